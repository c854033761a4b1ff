// Launches of the exact attention gradient (included by seq_bwd_*.hip).
#pragma once

#include <algorithm>

#include "seq_bwd.hpp"
#include "seq_host.hpp"

namespace ma_host {

template <typename T, int D, ma::Keys KEYS> int run_seq_bwd_d(Launcher &L, const ma::SeqBwd &p)
{
    const dim3 block(256);
    int rc = L.run(kSeqStats, [&] {
        return launched([&] { ma::seq_stats<T, KEYS><<<dim3((unsigned)p.stat_blocks), block, 0, L.stream>>>(p); });
    });
    if (rc != MA_OK) return rc;
    const int blocks_q = (int)((int64_t)p.tiles_q * p.pieces_q * p.Hkv), blocks_k = (int)((int64_t)p.tiles_k * p.pieces * p.Hkv);
    rc = L.run(kSeqBwd, [&] {
        return launched([&] { ma::seq_bwd<T, D, KEYS><<<dim3((unsigned)blocks_q + (unsigned)blocks_k), block, 0, L.stream>>>(p, blocks_q); });
    });
    if (rc != MA_OK || (p.pieces == 1 && p.pieces_q == 1)) return rc;
    // at most 8 workgroups a compute unit
    const int64_t rows = std::max((int64_t)(KEYS == ma::kCross ? p.keys : p.seqs).total * p.Hkv, p.pieces_q == 1 ? 0 : (int64_t)p.seqs.total * p.Hkv * p.G);
    const int64_t blocks = std::min<int64_t>(2048, (rows * (D / 4) + 255) / 256);
    return L.run(kSeqBwdJoin, [&] { return launched([&] { ma::seq_bwd_join<T, D, KEYS><<<dim3((unsigned)blocks), block, 0, L.stream>>>(p); }); });
}

template <typename T, ma::Keys KEYS> int run_seq_bwd_keys(Launcher &L, const ma::SeqBwd &p)
{
    switch (tile_d(p.d)) {
    case 64: return run_seq_bwd_d<T, 64, KEYS>(L, p);
    case 96: return run_seq_bwd_d<T, 96, KEYS>(L, p);
    default: return run_seq_bwd_d<T, 128, KEYS>(L, p);
    }
}

template <typename T> int run_seq_bwd_impl(Launcher &L, const ma::SeqBwd &p)
{
    return p.keys.cu ? run_seq_bwd_keys<T, ma::kCross>(L, p) : run_seq_bwd_keys<T, ma::kSelf>(L, p);
}

}  // namespace ma_host
