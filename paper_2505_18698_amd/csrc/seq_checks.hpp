// Argument checks that the C entry points over sequences, caches and beams share
// (seq_abi.hip, decoder_abi.hip).
#pragma once

#include <exception>

#include "seq_host.hpp"

namespace ma_host {

inline size_t elem_bytes(int32_t dtype) { return dtype == MA_F32 ? 4 : 2; }
inline size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

// A C function that cannot let a C++ exception out.
template <typename F> int guarded(F &&f)
{
    try {
        return f();
    } catch (const std::exception &e) {
        return fail(MA_ENOMEM, "out of host resources: %s", e.what());
    } catch (...) {
        return fail(MA_ENOMEM, "out of host resources");
    }
}

// A device memory range of an argument.
struct Range {
    const char *name;
    const void *p;
    size_t bytes;
};

inline int check_alignment(const Range &r, size_t to)
{
    if (!r.p) return fail(MA_EINVAL, "null %s pointer", r.name);
    if ((uintptr_t)r.p % to) return fail(MA_EINVAL, "%s must be %zu-byte aligned", r.name, to);
    return MA_OK;
}

// No output may overlap another one or an input.
template <size_t NO, size_t NI> int check_overlaps(const Range (&outs)[NO], const Range (&ins)[NI])
{
    for (size_t i = 0; i < NO; ++i) {
        if (!outs[i].p) continue;
        for (const Range &in : ins)
            if (in.p && ranges_overlap(outs[i].p, outs[i].bytes, in.p, in.bytes))
                return fail(MA_EINVAL, "%s must not overlap %s", outs[i].name, in.name);
        for (size_t j = i + 1; j < NO; ++j)
            if (outs[j].p && ranges_overlap(outs[i].p, outs[i].bytes, outs[j].p, outs[j].bytes))
                return fail(MA_EINVAL, "%s must not overlap %s", outs[i].name, outs[j].name);
    }
    return MA_OK;
}

constexpr int64_t kMaxWidth = int64_t(1) << 20;  // elements of a row: offsets within a tile of rows stay in 32 bits

inline int check_heads(int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int32_t dtype)
{
    if (dtype != MA_F32 && dtype != MA_BF16 && dtype != MA_F16) return fail(MA_EINVAL, "unknown dtype %d", dtype);
    if (B < 0 || total < 0) return fail(MA_EINVAL, "B and total must be >= 0");
    if (Hq < 1 || Hkv < 1 || d < 1) return fail(MA_EINVAL, "Hq, Hkv and d must be >= 1");
    if (Hq % Hkv) return fail(MA_EINVAL, "Hq (%lld) must be a multiple of Hkv (%lld)", (long long)Hq, (long long)Hkv);
    const int64_t chunk = 16 / (int64_t)elem_bytes(dtype);
    if (d > 128 || d % chunk)
        return fail(MA_EUNSUPPORTED, "d must be a multiple of %lld up to 128 (got %lld)", (long long)chunk, (long long)d);
    if (Hq > kMaxWidth / tile_d(d))
        return fail(MA_EUNSUPPORTED, "Hq times d, rounded up to %d, must not exceed %lld", (int)tile_d(d), (long long)kMaxWidth);
    if (B > 0x7ffffffe || total > 0x7fffff00 || total * (Hq / Hkv) > 0x7fffff00)
        return fail(MA_EUNSUPPORTED, "total * (Hq / Hkv) and B must be below 2^31");
    return MA_OK;
}

// Rows of `ld` elements that hold `width`.
inline int check_stride(const char *name, int64_t ld, int64_t width, int32_t dtype)
{
    const int64_t chunk = 16 / (int64_t)elem_bytes(dtype);
    if (ld < width || ld % chunk)
        return fail(MA_EINVAL, "%s (%lld) must be at least %lld and a multiple of %lld", name, (long long)ld, (long long)width,
                    (long long)chunk);
    if (ld > kMaxWidth) return fail(MA_EUNSUPPORTED, "%s must not exceed %lld", name, (long long)kMaxWidth);
    return MA_OK;
}

// (HIP launches fewer than 2^32 threads a dimension; every kernel here has kSeqThreads a workgroup.)
inline int check_grid(int64_t units, int64_t Hkv)
{
    if (units > 0xffffffffll / kSeqThreads / Hkv) return fail(MA_EUNSUPPORTED, "too many tiles for one grid");
    return MA_OK;
}

inline size_t span_bytes(int64_t rows, int64_t ld, int64_t width, int32_t dtype)
{
    return rows == 0 ? 0 : ((size_t)(rows - 1) * ld + width) * elem_bytes(dtype);
}

#define MA_TRY(x)                    \
    do {                             \
        const int rc_ = (x);         \
        if (rc_ != MA_OK) return rc_; \
    } while (0)

inline int check_pages(int64_t pages, int64_t page)
{
    if (page < 8 || page > 4096 || (page & (page - 1)))
        return fail(MA_EUNSUPPORTED, "page must be a power of two from 8 to 4096 (got %lld)", (long long)page);
    if (pages < 0 || pages > 0x7fffffff) return fail(MA_EINVAL, "pages must be in 0..2^31 - 1");
    return MA_OK;
}

// Bytes of the pages of K or of V, as far as any memory goes.
inline size_t cache_bytes(int64_t pages, int64_t Hkv, int64_t page, int64_t d, int32_t dtype)
{
    const unsigned __int128 n = (unsigned __int128)pages * Hkv * page * d * elem_bytes(dtype);
    return n >> 62 ? size_t(1) << 62 : (size_t)n;
}

inline int log2_of(int64_t page)
{
    int x = 0;
    while ((int64_t(1) << x) < page) ++x;
    return x;
}

// Alignment of the ranges that hold something and are not optional.
template <size_t N> int check_ranges(const Range (&r)[N], const size_t (&to)[N])
{
    for (size_t i = 0; i < N; ++i)
        if (r[i].bytes) MA_TRY(check_alignment(r[i], to[i]));
    return MA_OK;
}

}  // namespace ma_host
