// Launches of the exact attention gradient (included by seq_bwd_*.hip).
#pragma once

#include <algorithm>

#include "seq_bwd.hpp"
#include "seq_host.hpp"

namespace ma_host {

template <typename T, int D> int run_seq_bwd_d(Launcher &L, const ma::SeqBwd &p)
{
    const dim3 block(256);
    int rc = L.run(kSeqStats, [&] {
        return launched([&] { ma::seq_stats<T><<<dim3((unsigned)p.norm_blocks), block, 0, L.stream>>>(p); });
    });
    if (rc != MA_OK) return rc;
    rc = L.run(kSeqBwdK, [&] {
        return launched([&] { ma::seq_bwd_k<T, D><<<dim3((unsigned)((int64_t)p.tiles_k * p.pieces * p.Hkv)), dim3(ma::SeqBwdK<T, D>::NTH), 0, L.stream>>>(p); });
    });
    if (rc != MA_OK) return rc;
    if (p.pieces > 1) {
        // two rows' worth of threads at a time, at most 8 workgroups a compute unit
        const int64_t blocks = std::min<int64_t>(2048, ((int64_t)p.seqs.total * p.Hkv * (D / 4) + 255) / 256);
        rc = L.run(kSeqJoin, [&] { return launched([&] { ma::seq_bwd_join<T, D><<<dim3((unsigned)blocks), block, 0, L.stream>>>(p); }); });
        if (rc != MA_OK) return rc;
    }
    return L.run(kSeqBwdQ, [&] {
        return launched([&] { ma::seq_bwd_q<T, D><<<dim3((unsigned)((int64_t)p.tiles_q * p.Hkv)), block, 0, L.stream>>>(p); });
    });
}

template <typename T> int run_seq_bwd_impl(Launcher &L, const ma::SeqBwd &p)
{
    switch (tile_d(p.d)) {
    case 64: return run_seq_bwd_d<T, 64>(L, p);
    case 96: return run_seq_bwd_d<T, 96>(L, p);
    default: return run_seq_bwd_d<T, 128>(L, p);
    }
}

}  // namespace ma_host
