// Launches of the exact attention forward (included by seq_fwd_*.hip).
#pragma once

#include <algorithm>

#include "seq_attn.hpp"
#include "seq_host.hpp"

namespace ma_host {

template <typename T, int D> int run_seq_fwd_d(Launcher &L, const ma::SeqFwd &p, const SeqPlan &how)
{
    const dim3 grid((unsigned)(how.units * p.Hkv)), block(256);
    const bool few = how.rows == kSeqFewRows;
    constexpr int R = kSeqRows<T>, WR = R / 32;
    constexpr int kLds = 160 << 10;
    using ma::kCross, ma::kPaged, ma::kSelf;
    static_assert(std::min(2, kLds / ma::SeqAttn<T, D, 1, kPaged, true>::LDS_BYTES) == seq_residents<T>(D, true) &&
                      std::min(2, kLds / ma::SeqAttn<T, D, WR, kPaged, true>::LDS_BYTES) == seq_residents<T>(D, false),
                  "the shares of a split call are as many as the device holds");
    int rc = L.run(kSeqFwd, [&] {
        return launched([&] {
            auto by_rows = [&](auto keys) {
                constexpr ma::Keys K = decltype(keys)::value;
                if (!how.split && !few)
                    ma::seq_attention<T, D, WR, K, false><<<grid, block, 0, L.stream>>>(p);
                else if (!how.split)
                    ma::seq_attention<T, D, 1, K, false><<<grid, block, 0, L.stream>>>(p);
                else if (!few)
                    ma::seq_attention<T, D, WR, K, true><<<grid, block, 0, L.stream>>>(p);
                else
                    ma::seq_attention<T, D, 1, K, true><<<grid, block, 0, L.stream>>>(p);
            };
            if (how.keys == kSelf)
                ma::seq_attention<T, D, WR, kSelf, false><<<grid, block, 0, L.stream>>>(p);
            else if (how.keys == kPaged)
                by_rows(std::integral_constant<ma::Keys, kPaged>{});
            else
                by_rows(std::integral_constant<ma::Keys, kCross>{});
        });
    });
    if (rc != MA_OK || !how.split) return rc;
    const unsigned tiles = (unsigned)((int64_t)p.tiles * p.Hkv);
    return L.run(kSeqJoin, [&] {
        return launched([&] {
            if (few)
                ma::seq_join<T, D, kSeqFewRows><<<dim3(tiles, 8), block, 0, L.stream>>>(p);
            else
                ma::seq_join<T, D, R><<<dim3(tiles, R / 8), block, 0, L.stream>>>(p);
        });
    });
}

template <typename T> int run_seq_fwd_impl(Launcher &L, const ma::SeqFwd &p, const SeqPlan &how)
{
    switch (tile_d(p.d)) {
    case 64: return run_seq_fwd_d<T, 64>(L, p, how);
    case 96: return run_seq_fwd_d<T, 96>(L, p, how);
    default: return run_seq_fwd_d<T, 128>(L, p, how);
    }
}

}  // namespace ma_host
