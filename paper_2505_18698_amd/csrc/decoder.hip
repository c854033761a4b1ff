// Launches of the rotation, of the selection of beams and of the cache's reordering.
#include <algorithm>

#include "beam.hpp"
#include "decoder_host.hpp"
#include "rotary.hpp"

namespace ma_host {

template <typename T, int V, bool APPEND> static int run_rotate_as(Launcher &L, const ma::Rotate &p)
{
    const unsigned blocks = (unsigned)(((int64_t)p.seqs.total + p.rows - 1) / p.rows);
    return L.run(kRotate, [&] { return launched([&] { ma::rotate<T, V, APPEND><<<dim3(blocks), dim3(256), 0, L.stream>>>(p); }); });
}

// 16 bytes of both halves a thread where the halves are whole numbers of 16 bytes, else 8.
template <typename T> static int run_rotate_of(Launcher &L, const ma::Rotate &p, bool append)
{
    constexpr int V = 16 / (int)sizeof(T);
    if (p.rot % (2 * V) == 0) return append ? run_rotate_as<T, V, true>(L, p) : run_rotate_as<T, V, false>(L, p);
    if constexpr (sizeof(T) == 2) return append ? run_rotate_as<T, V / 2, true>(L, p) : run_rotate_as<T, V / 2, false>(L, p);
    return fail(MA_EUNSUPPORTED, "rot must be a multiple of 8");
}

int run_rotate(Launcher &L, const ma::Rotate &p, int32_t dtype, bool append)
{
    switch (dtype) {
    case MA_F32: return run_rotate_of<float>(L, p, append);
    case MA_BF16: return run_rotate_of<__bf16>(L, p, append);
    default: return run_rotate_of<_Float16>(L, p, append);
    }
}

int run_beam_select(Launcher &L, const ma::BeamSelect &p, int32_t dtype)
{
    const dim3 grid((unsigned)((int64_t)p.B * p.K * p.parts));
    const int rc = L.run(kBeamParts, [&] {
        return launched([&] {
            switch (dtype) {
            case MA_F32: ma::beam_parts<float><<<grid, dim3(256), 0, L.stream>>>(p); break;
            case MA_BF16: ma::beam_parts<__bf16><<<grid, dim3(256), 0, L.stream>>>(p); break;
            default: ma::beam_parts<_Float16><<<grid, dim3(256), 0, L.stream>>>(p); break;
            }
        });
    });
    if (rc != MA_OK) return rc;
    const size_t lds = ((size_t)p.K * p.parts + 8) * sizeof(ma::BeamHead);
    return L.run(kBeamJoin, [&] { return launched([&] { ma::beam_join<<<dim3((unsigned)p.B), dim3(256), lds, L.stream>>>(p); }); });
}

int run_paged_reorder(Launcher &L, const ma::PagedReorder &p)
{
    // the longest a started page can be, 16 bytes a thread, and as many entries of a table
    const int64_t most = 2ll * p.Hkv * ((1 << p.page_log2) - 1) * p.chunks;
    const int pages = (int)std::min<int64_t>((most + 255) / 256, 4096), tables = p.move_table ? (int)std::min<int64_t>((p.blocks + 255) / 256, 64) : 0;
    const dim3 grid((unsigned)(pages + tables), (unsigned)p.B), block(256);
    return L.run(kReorder, [&] {
        return launched([&] {
            if (p.K <= 4) ma::paged_reorder<4><<<grid, block, 0, L.stream>>>(p, pages);
            else if (p.K <= 8) ma::paged_reorder<8><<<grid, block, 0, L.stream>>>(p, pages);
            else if (p.K <= 16) ma::paged_reorder<16><<<grid, block, 0, L.stream>>>(p, pages);
            else ma::paged_reorder<32><<<grid, block, 0, L.stream>>>(p, pages);
        });
    });
}

}  // namespace ma_host
