// C ABI of the exact attention over packed sequences and paged caches
// (include/monarch_attn.h): argument checks, workspaces and how a call runs.
#include <algorithm>
#include <cmath>
#include <exception>

#include "seq_host.hpp"
#include "seq_params.hpp"

namespace {

using namespace ma_host;

size_t elem_bytes(int32_t dtype) { return dtype == MA_F32 ? 4 : 2; }
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }

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

int check_alignment(const Range &r, size_t to)
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

int check_heads(int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int32_t dtype)
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
int check_stride(const char *name, int64_t ld, int64_t width, int32_t dtype)
{
    const int64_t chunk = 16 / (int64_t)elem_bytes(dtype);
    if (ld < width || ld % chunk)
        return fail(MA_EINVAL, "%s (%lld) must be at least %lld and a multiple of %lld", name, (long long)ld, (long long)width,
                    (long long)chunk);
    if (ld > kMaxWidth) return fail(MA_EUNSUPPORTED, "%s must not exceed %lld", name, (long long)kMaxWidth);
    return MA_OK;
}

// Row tiles of R packed rows over all sequences, at most (tile0 in seq_tiles.hpp), and one without
// any.
int64_t tiles_of(int64_t total, int64_t rows_a_token, int64_t B, int64_t R) { return std::max<int64_t>(1, total * rows_a_token / R + B); }

// (HIP launches fewer than 2^32 threads a dimension; every kernel here has kSeqThreads a workgroup.)
int check_grid(int64_t units, int64_t Hkv)
{
    if (units > 0xffffffffll / kSeqThreads / Hkv) return fail(MA_EUNSUPPORTED, "too many tiles for one grid");
    return MA_OK;
}

float log2_scale(int64_t d) { return (float)(1.4426950408889634 / std::sqrt((double)d)); }

size_t span_bytes(int64_t rows, int64_t ld, int64_t width, int32_t dtype)
{
    return rows == 0 ? 0 : ((size_t)(rows - 1) * ld + width) * elem_bytes(dtype);
}

#define MA_TRY(x)                    \
    do {                             \
        const int rc_ = (x);         \
        if (rc_ != MA_OK) return rc_; \
    } while (0)

struct FwdLaunch {
    ma::SeqFwd p;
    SeqPlan how;
    int32_t dtype;
    static int run(Launcher &L, void *a)
    {
        const FwdLaunch &x = *(const FwdLaunch *)a;
        switch (x.dtype) {
        case MA_F32: return run_seq_fwd<float>(L, x.p, x.how);
        case MA_BF16: return run_seq_fwd<__bf16>(L, x.p, x.how);
        default: return run_seq_fwd<_Float16>(L, x.p, x.how);
        }
    }
};

struct BwdLaunch {
    ma::SeqBwd p;
    int32_t dtype;
    static int run(Launcher &L, void *a)
    {
        const BwdLaunch &x = *(const BwdLaunch *)a;
        switch (x.dtype) {
        case MA_F32: return run_seq_bwd<float>(L, x.p);
        case MA_BF16: return run_seq_bwd<__bf16>(L, x.p);
        default: return run_seq_bwd<_Float16>(L, x.p);
        }
    }
};

int packed_fwd(const void *q, const void *k, const void *v, void *out, float *lse, void *rest, const int32_t *cu, int64_t B,
               int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t ldk, int64_t ldv, int32_t causal,
               int32_t clear, int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_heads(B, total, Hq, Hkv, d, dtype));
    MA_TRY(check_stride("ldq", ldq, Hq * d, dtype));
    MA_TRY(check_stride("ldk", ldk, Hkv * d, dtype));
    MA_TRY(check_stride("ldv", ldv, Hkv * d, dtype));
    const int64_t G = Hq / Hkv, tiles = tiles_of(total, G, B, seq_rows(dtype));
    MA_TRY(check_grid(tiles, Hkv));
    if (total == 0 || (B == 0 && !clear)) return MA_OK;  // nothing to compute: no launch, no pointer read
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k", k, span_bytes(total, ldk, Hkv * d, dtype)},
                         {"v", v, span_bytes(total, ldv, Hkv * d, dtype)},
                         {"cu_seqlens", cu, (size_t)(B + 1) * 4}};
    const size_t ob = span_bytes(total, Hq * d, Hq * d, dtype);
    const Range outs[] = {{"out", out, ob}, {"lse", lse, (size_t)(Hq * total) * 4}, {"rest", rest, ob}};
    if (rest && dtype == MA_F32) return fail(MA_EINVAL, "rest is of 16-bit outputs");
    for (int i = 0; i < 4; ++i) MA_TRY(check_alignment(ins[i], i < 3 ? 16 : 4));
    MA_TRY(check_alignment(outs[0], 16));
    if (lse) MA_TRY(check_alignment(outs[1], 4));
    if (rest) MA_TRY(check_alignment(outs[2], 16));
    MA_TRY(check_overlaps(outs, ins));
    FwdLaunch x{};
    ma::SeqFwd &p = x.p;
    p.q = q, p.k = k, p.v = v, p.out = out, p.lse = lse, p.rest = rest;
    p.seqs = ma::Seqs{cu, (int)B, (int)total};
    p.Hkv = (int)Hkv, p.G = (int)G, p.d = (int)d;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv;
    p.c = log2_scale(d), p.causal = causal != 0, p.clear = clear != 0, p.tiles = (int)tiles;
    x.how = SeqPlan{false, false, seq_rows(dtype), tiles};
    x.dtype = dtype;
    return run_launches(stream, FwdLaunch::run, &x);
}

// Workspace of the gradient: lse in log2 units and delta of every row and head; in fp16 also the
// norms of the rows of dout and v.
constexpr int kStatBlocks = 1024;
size_t stat_bytes_of(int64_t total, int64_t heads) { return align_up((size_t)(heads * total) * 4); }
size_t bwd_bytes(int64_t total, int64_t Hq, int64_t Hkv, int32_t dtype)
{
    return (dtype == MA_F16 ? 3 : 2) * stat_bytes_of(total, Hq) + (dtype == MA_F16 ? stat_bytes_of(total, Hkv) : 0);
}

// Pieces that the query rows of a key tile are cut into, all those of a call alike.  The longest
// walk, of the first keys of one causal sequence that fills the call, is twice the mean one, so 1024
// key tiles and heads (two rounds of two workgroups on 256 compute units) end with it; the pieces
// make it half of the mean work of a compute unit's slot.  More than three are not worth their sums'
// way through memory (9550 rows, 16 heads on 4 of 128, with the forward: 608 us; 614 with two or
// four), nor are any where even one sequence of all the call's rows would be a walk of fewer than 16
// tiles (dQ, dK, dV and the sums of 64 sequences of 10, 4 heads of 64: 9 us, 16 with three pieces).
//
// The host knows the rows and not the lengths. So short sequences that are many pay for the pieces
// that one long one among them would need: 6 of 1 to 1000 tokens, 12 heads of 64 in fp32, take 95 us
// with three pieces and 112 with one, but 64 of 100, 16 heads on 4 of 128, 87 and 63 us.
int64_t bwd_pieces(int64_t total, int64_t tiles_k, int64_t Hkv, int64_t G, int64_t num_cus)
{
    const int64_t want = (8 * num_cus + tiles_k * Hkv - 1) / (tiles_k * Hkv);
    const int64_t longest = G * ((total + kSeqBwdKeys - 1) / kSeqBwdKeys);
    return std::max<int64_t>(1, std::min<int64_t>({want, 3, longest / 8}));
}

int packed_bwd(const void *q, const void *k, const void *v, const void *out, const float *lse, const void *rest,
               const void *dout, void *dq, void *dk, void *dv, const int32_t *cu, int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d,
               int64_t ldq, int64_t ldk, int64_t ldv, int32_t causal, int32_t clear, int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_heads(B, total, Hq, Hkv, d, dtype));
    MA_TRY(check_stride("ldq", ldq, Hq * d, dtype));
    MA_TRY(check_stride("ldk", ldk, Hkv * d, dtype));
    MA_TRY(check_stride("ldv", ldv, Hkv * d, dtype));
    const int64_t G = Hq / Hkv, tiles_q = tiles_of(total, G, B, seq_rows(dtype)), tiles_k = tiles_of(total, 1, B, kSeqBwdKeys);
    MA_TRY(check_grid(std::max(tiles_q, tiles_k), Hkv));
    if (total == 0 || (B == 0 && !clear)) return MA_OK;
    const size_t qb = span_bytes(total, Hq * d, Hq * d, dtype), kb = span_bytes(total, Hkv * d, Hkv * d, dtype);
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k", k, span_bytes(total, ldk, Hkv * d, dtype)},
                         {"v", v, span_bytes(total, ldv, Hkv * d, dtype)},
                         {"out", out, qb},
                         {"dout", dout, qb},
                         {"lse", lse, (size_t)(Hq * total) * 4},
                         {"cu_seqlens", cu, (size_t)(B + 1) * 4},
                         {"rest", rest, qb}};
    if (rest && dtype == MA_F32) return fail(MA_EINVAL, "rest is of 16-bit outputs");
    const Range outs[] = {{"dq", dq, qb}, {"dk", dk, kb}, {"dv", dv, kb}};
    for (int i = 0; i < 7; ++i) MA_TRY(check_alignment(ins[i], i < 5 ? 16 : 4));
    if (rest) MA_TRY(check_alignment(ins[7], 16));
    for (const Range &r : outs) MA_TRY(check_alignment(r, 16));
    MA_TRY(check_overlaps(outs, ins));
    CallScope c;
    MA_TRY(begin_call(c));
    const int64_t pieces = bwd_pieces(total, tiles_k, Hkv, G, c.num_cus);
    const size_t part = pieces > 1 ? (size_t)(pieces * total * Hkv) * tile_d(d) * 4 : 0, stat_bytes = bwd_bytes(total, Hq, Hkv, dtype);
    MA_TRY(check_grid(tiles_k * pieces + tiles_q, Hkv));
    MA_TRY(call_workspace(stream, stat_bytes + 2 * part, c));
    BwdLaunch x{};
    ma::SeqBwd &p = x.p;
    p.q = q, p.k = k, p.v = v, p.out = out, p.dout = dout, p.lse = lse, p.rest = rest;
    p.dq = dq, p.dk = dk, p.dv = dv;
    p.seqs = ma::Seqs{cu, (int)B, (int)total};
    p.Hkv = (int)Hkv, p.G = (int)G, p.d = (int)d;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv;
    p.c = log2_scale(d), p.causal = causal != 0, p.clear = clear != 0;
    p.tiles_q = (int)tiles_q, p.tiles_k = (int)tiles_k;
    const size_t each = stat_bytes_of(total, Hq);
    p.lse2 = (float *)c.ws, p.delta = (float *)(c.ws + each);
    if (dtype == MA_F16) p.norm_g = (float *)(c.ws + 2 * each), p.norm_v = (float *)(c.ws + 3 * each);
    p.stat_blocks = (int)std::min<int64_t>(kStatBlocks, (total + 15) / 16 * Hq);
    p.pieces = (int)pieces;
    p.part_k = (float *)(c.ws + stat_bytes), p.part_v = (float *)(c.ws + stat_bytes + part);
    x.dtype = dtype;
    return run_launches(stream, BwdLaunch::run, &x);
}

int check_pages(int64_t pages, int64_t page)
{
    if (page < 8 || page > 4096 || (page & (page - 1)))
        return fail(MA_EUNSUPPORTED, "page must be a power of two from 8 to 4096 (got %lld)", (long long)page);
    if (pages < 0 || pages > 0x7fffffff) return fail(MA_EINVAL, "pages must be in 0..2^31 - 1");
    return MA_OK;
}

int log2_of(int64_t page)
{
    int x = 0;
    while ((int64_t(1) << x) < page) ++x;
    return x;
}

// How a paged call runs.  Sequences of few new rows (on average no more than 32 packed ones: single
// tokens) take 32-row tiles, whose waves share the keys. The work is shared evenly by as many
// workgroups as the device holds at a time (seq_residents; find_share in seq_attn.hpp), except
// where the keys of the longest possible context take no more than kWholeBytes, or where tiles of many
// rows are 16 times as many: then a row tile is a workgroup's. (64 single tokens over up to
// 8192: 103 us, in pieces of equal length 122, 128-row tiles 266; 8 chunks of up to 512 over up to
// 16384, before the copies' addresses were found in lanes: 213 us, in pieces of equal length 241.
// With two workgroups a compute unit that holds one: 64 tokens over up to 8192, fp32, 32 heads on 8
// of 64, 292 us for 285; 2 chunks of 100 over 5000, fp32, 16 on 4 of 128, 131 us for 117. Many row
// tiles, a tile a workgroup and in shares, heads of 128 in bf16: 128 chunks of 512 over 2000 to 4000,
// 32 heads on 8: 3.0 and 4.7 ms; single tokens of 1100 requests over 300, the same heads: 440 and 289 us,
// over 1000 and one over 100000: 2.29 and 0.85 ms; of 600 over 500, fp32, 16 heads of 64: 731 and 780 us.)
//
// kWholeBytes: one token over 500 and 1000, 4 heads of 64: 9 and 12 us whole, 14 split; 8 heads of
// 128: 13 and 18 us whole, 15 split.
constexpr int64_t kWholeBytes = 128 << 10;
struct PagedSplit {
    int rows;
    bool split;
    int64_t tiles, units;
    size_t bytes_o, bytes_l, bytes_parts;
};

// Packed rows a workgroup takes.
int paged_rows(int64_t total, int64_t B, int64_t G, int32_t dtype) { return total * G <= B * kSeqFewRows ? kSeqFewRows : seq_rows(dtype); }

PagedSplit paged_split(int64_t total, int64_t B, int64_t G, int64_t Hkv, int64_t d, int64_t max_keys, int64_t num_cus, int32_t dtype)
{
    PagedSplit s{paged_rows(total, B, G, dtype), false, 0, 0, 0, 0, 0};
    s.tiles = s.units = tiles_of(total, G, B, s.rows);
    const bool few = s.rows == kSeqFewRows;
    const int64_t shares = std::max<int64_t>(1, seq_residents(dtype, d, few) * num_cus / Hkv);
    if ((!few && s.tiles >= 16 * shares) || max_keys * tile_d(d) * (int64_t)elem_bytes(dtype) <= kWholeBytes) return s;
    s.split = true;
    s.units = shares;
    const size_t rows = (size_t)(2 * shares) * Hkv * s.rows;  // two segments a share (find_share in seq_attn.hpp)
    s.bytes_o = align_up(rows * tile_d(d) * 4);
    s.bytes_l = align_up(rows * 4);
    s.bytes_parts = align_up((size_t)(s.tiles + 1) * sizeof(ma::SeqTileParts));
    return s;
}

int paged_fwd(const void *q, const void *k_pages, const void *v_pages, void *out, float *lse, const int32_t *cu,
              const int32_t *kv_lens, const int32_t *table, int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d,
              int64_t ldq, int64_t pages, int64_t page, int64_t blocks, int32_t causal, int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_heads(B, total, Hq, Hkv, d, dtype));
    MA_TRY(check_stride("ldq", ldq, Hq * d, dtype));
    MA_TRY(check_pages(pages, page));
    if (blocks < 0 || blocks > 0x7fffffff) return fail(MA_EINVAL, "blocks must be in 0..2^31 - 1");
    const int64_t G = Hq / Hkv;
    MA_TRY(check_grid(tiles_of(total, G, B, paged_rows(total, B, G, dtype)), Hkv));
    if (B == 0 || total == 0) return MA_OK;
    const size_t cache = (size_t)pages * Hkv * page * d * elem_bytes(dtype);
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k_pages", k_pages, cache},
                         {"v_pages", v_pages, cache},
                         {"cu_seqlens", cu, (size_t)(B + 1) * 4},
                         {"kv_lens", kv_lens, (size_t)B * 4},
                         {"block_table", table, (size_t)B * blocks * 4}};
    const Range outs[] = {{"out", out, span_bytes(total, Hq * d, Hq * d, dtype)}, {"lse", lse, (size_t)(Hq * total) * 4}};
    for (int i = 0; i < 6; ++i) {
        if ((i == 1 || i == 2) && pages == 0) continue;  // an empty cache and an empty table are never read
        if (i == 5 && blocks == 0) continue;
        MA_TRY(check_alignment(ins[i], i < 3 ? 16 : 4));
    }
    MA_TRY(check_alignment(outs[0], 16));
    if (lse) MA_TRY(check_alignment(outs[1], 4));
    MA_TRY(check_overlaps(outs, ins));
    CallScope c;
    MA_TRY(begin_call(c));
    const PagedSplit s = paged_split(total, B, G, Hkv, d, blocks * page, c.num_cus, dtype);
    if (s.split) {
        MA_TRY(check_grid(s.units, Hkv));
        MA_TRY(call_workspace(stream, s.bytes_o + s.bytes_l + s.bytes_parts, c));
    }
    FwdLaunch x{};
    ma::SeqFwd &p = x.p;
    p.q = q, p.k = k_pages, p.v = v_pages, p.out = out, p.lse = lse;
    p.seqs = ma::Seqs{cu, (int)B, (int)total};
    p.kv_lens = kv_lens, p.table = table;
    p.Hkv = (int)Hkv, p.G = (int)G, p.d = (int)d;
    p.ldq = ldq;
    p.page_log2 = log2_of(page), p.pages = (int)pages, p.blocks = (int)blocks;
    p.c = log2_scale(d), p.causal = causal != 0, p.tiles = (int)s.tiles;
    p.part_o = (float *)c.ws, p.part_l = (float *)(c.ws + s.bytes_o);
    p.parts = (ma::SeqTileParts *)(c.ws + s.bytes_o + s.bytes_l);
    p.shares = (int)s.units;
    x.how = SeqPlan{true, s.split, s.rows, s.units};
    x.dtype = dtype;
    return run_launches(stream, FwdLaunch::run, &x);
}

int paged_plan(const int32_t *past, const int32_t *fresh, const int32_t *ring, const int32_t *free_in, int32_t *table,
               int32_t *cu, int32_t *kv_lens, int64_t *slots, int32_t *free_out, int32_t *status, int64_t B,
               int64_t ring_len, int64_t blocks, int64_t page, int64_t capacity, hipStream_t stream)
{
    MA_TRY(check_pages(0, page));
    if (B < 0 || ring_len < 0 || blocks < 0 || capacity < 0)
        return fail(MA_EINVAL, "B, ring_len, blocks and capacity must be >= 0");
    if (B > MONARCH_ATTN_PLAN_MAX_B) return fail(MA_EUNSUPPORTED, "B must be <= %d (got %lld)", MONARCH_ATTN_PLAN_MAX_B, (long long)B);
    if (ring_len > 0x7fffffff || blocks > 0x7fffffff || capacity > 0x7fffff00)
        return fail(MA_EUNSUPPORTED, "ring_len, blocks and capacity must be below 2^31");
    const Range ins[] = {{"past", past, (size_t)B * 4}, {"fresh", fresh, (size_t)B * 4}, {"ring", ring, (size_t)ring_len * 4},
                         {"free_in", free_in, 8}};
    const Range outs[] = {{"block_table", table, (size_t)(B * blocks) * 4}, {"cu_seqlens", cu, (size_t)(B + 1) * 4},
                          {"kv_lens", kv_lens, (size_t)B * 4}, {"slots", slots, (size_t)capacity * 8},
                          {"free_out", free_out, 8}, {"status", status, 4}};
    for (const Range &r : ins)
        if (r.bytes) MA_TRY(check_alignment(r, 4));
    for (const Range &r : outs)
        if (r.bytes) MA_TRY(check_alignment(r, &r == &outs[3] ? 8 : 4));
    MA_TRY(check_overlaps(outs, ins));
    ma::PagedPlan p{past, fresh, ring, free_in, table, cu, kv_lens, slots, free_out, status, (int)B, (int)ring_len,
                    (int)blocks, log2_of(page), (int)capacity};
    return run_launches(stream, [](Launcher &L, void *a) { return run_paged_plan(L, *(const ma::PagedPlan *)a); }, &p);
}

int paged_write(const void *k, const void *v, void *k_pages, void *v_pages, const int64_t *slots, int64_t rows, int64_t Hkv,
                int64_t d, int64_t ldk, int64_t ldv, int64_t pages, int64_t page, int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_heads(1, rows, Hkv, Hkv, d, dtype));
    MA_TRY(check_stride("ldk", ldk, Hkv * d, dtype));
    MA_TRY(check_stride("ldv", ldv, Hkv * d, dtype));
    MA_TRY(check_pages(pages, page));
    const int64_t per = paged_write_rows(Hkv * d * (int64_t)elem_bytes(dtype) / 16);
    MA_TRY(check_grid((rows + per - 1) / per, 1));
    if (rows == 0 || pages == 0) return MA_OK;
    const size_t cache = (size_t)pages * Hkv * page * d * elem_bytes(dtype);
    const Range ins[] = {{"k", k, span_bytes(rows, ldk, Hkv * d, dtype)}, {"v", v, span_bytes(rows, ldv, Hkv * d, dtype)},
                         {"slots", slots, (size_t)rows * 8}};
    const Range outs[] = {{"k_pages", k_pages, cache}, {"v_pages", v_pages, cache}};
    for (int i = 0; i < 3; ++i) MA_TRY(check_alignment(ins[i], i < 2 ? 16 : 8));
    for (const Range &r : outs) MA_TRY(check_alignment(r, 16));
    MA_TRY(check_overlaps(outs, ins));
    ma::PagedWrite p{k, v, k_pages, v_pages, slots, (int)rows, (int)Hkv, (int)d, log2_of(page), (int)pages,
                     (int)elem_bytes(dtype), ldk, ldv};
    return run_launches(stream, [](Launcher &L, void *a) { return run_paged_write(L, *(const ma::PagedWrite *)a); }, &p);
}

}  // namespace

extern "C" {

int monarch_attn_exact_packed_fwd(const void *q, const void *k, const void *v, void *out, float *lse, void *rest,
                                  const int32_t *cu_seqlens, int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t ldk,
                                  int64_t ldv, int32_t causal, int32_t clear, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return packed_fwd(q, k, v, out, lse, rest, cu_seqlens, B, total, Hq, Hkv, d, ldq, ldk, ldv, causal, clear, dtype, (hipStream_t)stream);
    });
}

int monarch_attn_exact_packed_bwd(const void *q, const void *k, const void *v, const void *out, const float *lse,
                                  const void *rest, const void *dout, void *dq, void *dk, void *dv, const int32_t *cu_seqlens, int64_t B,
                                  int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t ldk, int64_t ldv,
                                  int32_t causal, int32_t clear, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return packed_bwd(q, k, v, out, lse, rest, dout, dq, dk, dv, cu_seqlens, B, total, Hq, Hkv, d, ldq, ldk, ldv, causal, clear, dtype,
                          (hipStream_t)stream);
    });
}

int monarch_attn_exact_paged_fwd(const void *q, const void *k_pages, const void *v_pages, void *out, float *lse,
                                 const int32_t *cu_seqlens, const int32_t *kv_lens, const int32_t *block_table, int64_t B,
                                 int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t pages, int64_t page,
                                 int64_t blocks, int32_t causal, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return paged_fwd(q, k_pages, v_pages, out, lse, cu_seqlens, kv_lens, block_table, B, total, Hq, Hkv, d, ldq, pages, page,
                         blocks, causal, dtype, (hipStream_t)stream);
    });
}

int monarch_attn_paged_plan(const int32_t *past, const int32_t *fresh, const int32_t *ring, const int32_t *free_in,
                            int32_t *block_table, int32_t *cu_seqlens, int32_t *kv_lens, int64_t *slots, int32_t *free_out,
                            int32_t *status, int64_t B, int64_t ring_len, int64_t blocks, int64_t page, int64_t capacity,
                            void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return paged_plan(past, fresh, ring, free_in, block_table, cu_seqlens, kv_lens, slots, free_out, status, B, ring_len,
                          blocks, page, capacity, (hipStream_t)stream);
    });
}

int monarch_attn_paged_write(const void *k, const void *v, void *k_pages, void *v_pages, const int64_t *slots, int64_t rows,
                             int64_t Hkv, int64_t d, int64_t ldk, int64_t ldv, int64_t pages, int64_t page, int32_t dtype,
                             void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return paged_write(k, v, k_pages, v_pages, slots, rows, Hkv, d, ldk, ldv, pages, page, dtype, (hipStream_t)stream);
    });
}

}  // extern "C"
