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
    static_assert(std::min(2, kLds / ma::SeqAttn<T, D, 1, true, true>::LDS_BYTES) == seq_residents<T>(D, true) &&
                      std::min(2, kLds / ma::SeqAttn<T, D, WR, true, true>::LDS_BYTES) == seq_residents<T>(D, false),
                  "the shares of a split call are as many as the device holds");
    int rc = L.run(kSeqFwd, [&] {
        return launched([&] {
            if (!how.paged)
                ma::seq_attention<T, D, WR, false, false><<<grid, block, 0, L.stream>>>(p);
            else if (!how.split && !few)
                ma::seq_attention<T, D, WR, true, false><<<grid, block, 0, L.stream>>>(p);
            else if (!how.split)
                ma::seq_attention<T, D, 1, true, false><<<grid, block, 0, L.stream>>>(p);
            else if (!few)
                ma::seq_attention<T, D, WR, true, true><<<grid, block, 0, L.stream>>>(p);
            else
                ma::seq_attention<T, D, 1, true, true><<<grid, block, 0, L.stream>>>(p);
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
