// C ABI of the exact attention over packed sequences, paged caches and other sequences' rows
// (include/monarch_attn.h): argument checks, workspaces and how a call runs.
#include <algorithm>
#include <cmath>

#include "seq_checks.hpp"
#include "seq_params.hpp"

namespace {

using namespace ma_host;

// Row tiles of R packed rows over all sequences, at most (tile0 in seq_tiles.hpp), and one without
// any.
int64_t tiles_of(int64_t total, int64_t rows_a_token, int64_t B, int64_t R) { return std::max<int64_t>(1, total * rows_a_token / R + B); }

float log2_scale(int64_t d) { return (float)(1.4426950408889634 / std::sqrt((double)d)); }

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
    x.how = SeqPlan{ma::kSelf, false, seq_rows(dtype), tiles};
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
    p.pieces = (int)pieces, p.pieces_q = 1;
    p.part_k = (float *)(c.ws + stat_bytes), p.part_v = (float *)(c.ws + stat_bytes + part);
    x.dtype = dtype;
    return run_launches(stream, BwdLaunch::run, &x);
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
    const size_t cache = cache_bytes(pages, Hkv, page, d, dtype);
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
    x.how = SeqPlan{ma::kPaged, s.split, s.rows, s.units};
    x.dtype = dtype;
    return run_launches(stream, FwdLaunch::run, &x);
}

// The split of a cross call: that of a paged one, by the mean number of keys, which is what the host
// knows of them (of a padded batch half the width).  Many rows, whose steps take longer, are split from a quarter
// of that on where there are few tiles of them for the device, or few for long walks.  (Whole and split, bf16. Four rows a sequence, 12 heads of 64: 32
// sequences of 300 to 500 keys 12 and 19 us, of 100 to 1500 18 and 24. Many rows: 12 sequences of up to 400
// rows over up to 1500 keys, 16 heads on 4 of 128: 40 and 47 us; 24 of up to 512 over up to 2048, 12 heads of
// 64: 39 and 43; 64 of up to 512 over up to 1000, 16 heads: 115 and 138; 8 of up to 1024 over up to 8192, 16 heads on 4
// of 128: 174 and 137; 512 over 8192: 130 and 55. fp32, 16 of up to 300 over up to 1000, 12 heads of 64: 83 and 67.)
PagedSplit cross_split(int64_t total, int64_t total_k, bool padded, int64_t B, int64_t G, int64_t Hkv, int64_t d, int64_t num_cus, int32_t dtype)
{
    const int64_t mean = (total_k + std::max<int64_t>(1, B) - 1) / std::max<int64_t>(1, B) / (padded ? 2 : 1);
    const bool few = paged_rows(total, B, G, dtype) == kSeqFewRows;
    PagedSplit s = paged_split(total, B, G, Hkv, d, few ? mean : std::min(total_k, 4 * mean), num_cus, dtype);
    const bool long_walks = mean > (dtype == MA_F32 ? 128 : 1024);
    if (s.split && !few && 4 * s.tiles >= (long_walks ? 8 : 3) * s.units) s.split = false, s.units = s.tiles;
    return s;
}

int check_cross(int64_t B, int64_t total, int64_t total_k, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t ldk,
                int64_t ldv, int32_t dtype)
{
    MA_TRY(check_heads(B, total, Hq, Hkv, d, dtype));
    if (total_k < 0) return fail(MA_EINVAL, "total_k must be >= 0");
    if (total_k > 0x7fffff00) return fail(MA_EUNSUPPORTED, "total_k must be below 2^31");
    MA_TRY(check_stride("ldq", ldq, Hq * d, dtype));
    MA_TRY(check_stride("ldk", ldk, Hkv * d, dtype));
    return check_stride("ldv", ldv, Hkv * d, dtype);
}

int cross_fwd(const void *q, const void *k, const void *v, void *out, float *lse, void *rest, const int32_t *cu_q,
              const int32_t *cu_k, const int32_t *k_lens, int64_t B, int64_t total, int64_t total_k, int64_t Hq, int64_t Hkv,
              int64_t d, int64_t ldq, int64_t ldk, int64_t ldv, int32_t clear, int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_cross(B, total, total_k, Hq, Hkv, d, ldq, ldk, ldv, dtype));
    const int64_t G = Hq / Hkv;
    MA_TRY(check_grid(tiles_of(total, G, B, paged_rows(total, B, G, dtype)), Hkv));
    if (total == 0 || (B == 0 && !clear)) return MA_OK;
    if (rest && dtype == MA_F32) return fail(MA_EINVAL, "rest is of 16-bit outputs");
    const size_t ob = span_bytes(total, Hq * d, Hq * d, dtype), starts = (size_t)(B + 1) * 4;
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k", k, span_bytes(total_k, ldk, Hkv * d, dtype)},
                         {"v", v, span_bytes(total_k, ldv, Hkv * d, dtype)},
                         {"cu_q", cu_q, starts},
                         {"cu_k", cu_k, starts},
                         {"k_lens", k_lens, k_lens ? (size_t)B * 4 : 0}};
    const Range outs[] = {{"out", out, ob}, {"lse", lse, lse ? (size_t)(Hq * total) * 4 : 0}, {"rest", rest, rest ? ob : 0}};
    MA_TRY(check_ranges(ins, {16, 16, 16, 4, 4, 4}));
    MA_TRY(check_ranges(outs, {16, 4, 16}));
    MA_TRY(check_overlaps(outs, ins));
    CallScope c;
    MA_TRY(begin_call(c));
    PagedSplit s = cross_split(total, total_k, k_lens != nullptr, B, G, Hkv, d, c.num_cus, dtype);
    if (s.split && B > 0) {
        MA_TRY(check_grid(s.units, Hkv));
        MA_TRY(call_workspace(stream, s.bytes_o + s.bytes_l + s.bytes_parts, c));
    } else {
        s.split = false, s.units = s.tiles;
    }
    FwdLaunch x{};
    ma::SeqFwd &p = x.p;
    p.q = q, p.k = k, p.v = v, p.out = out, p.lse = lse, p.rest = rest;
    p.seqs = ma::Seqs{cu_q, (int)B, (int)total};
    p.keys = ma::KeySeqs{{cu_k, (int)B, (int)total_k}, k_lens};
    p.Hkv = (int)Hkv, p.G = (int)G, p.d = (int)d;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv;
    p.c = log2_scale(d), p.clear = clear != 0, p.tiles = (int)s.tiles;
    p.part_o = (float *)c.ws, p.part_l = (float *)(c.ws + s.bytes_o);
    p.parts = (ma::SeqTileParts *)(c.ws + s.bytes_o + s.bytes_l);
    p.shares = (int)s.units;
    x.how = SeqPlan{ma::kCross, s.split, s.rows, s.units};
    x.dtype = dtype;
    return run_launches(stream, FwdLaunch::run, &x);
}

// Pieces of the walks of a cross call's gradient. A key tile walks the rows of its sequence, a row tile the
// keys, in steps of 4 and 3 products: where the mean walk is longer than what a workgroup's share of all steps
// is (two workgroups a compute unit), it is cut.  (bf16, the whole gradient: 512 rows of 16 heads on 4 of 128
// over 8192 keys: 151 us, dQ in one piece 182, in 8 144; 2 sequences of 4096 rows over up to 512 keys: 150 us
// with 8 pieces of dK and dV, 186 with 4, 520 with one; 8 of up to 1024 over up to 8192: 400 us in one piece each, 430 in two.)
struct CrossPieces {
    int64_t keys, rows;
};
CrossPieces cross_pieces(int64_t B, int64_t total, int64_t total_k, int64_t tiles_q, int64_t tiles_k, int64_t Hkv, int64_t G, int64_t num_cus)
{
    const double n = std::max<int64_t>(1, B), walk_k = 4.0 * (double)G * total / n / kSeqBwdKeys, walk_q = 3.0 * total_k / n / kSeqBwdKeys;
    const double share = (walk_k * tiles_k + walk_q * tiles_q) * Hkv / (2.0 * num_cus);
    // (no sums to cut where a walk's own side has no rows: their join would be a launch of no workgroup)
    auto cut = [&](double walk, int64_t rows) { return rows == 0 ? 1 : (int64_t)std::max(1.0, std::min(8.0, std::ceil(walk / std::max(share, 16.0)))); };
    return CrossPieces{cut(walk_k, total_k), cut(walk_q, total)};
}

int cross_bwd(const void *q, const void *k, const void *v, const void *out, const float *lse, const void *rest, const void *dout,
              void *dq, void *dk, void *dv, const int32_t *cu_q, const int32_t *cu_k, const int32_t *k_lens, int64_t B, int64_t total,
              int64_t total_k, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t ldk, int64_t ldv, int32_t clear, int32_t dtype,
              hipStream_t stream)
{
    MA_TRY(check_cross(B, total, total_k, Hq, Hkv, d, ldq, ldk, ldv, dtype));
    const int64_t G = Hq / Hkv, tiles_q = tiles_of(total, G, B, seq_rows(dtype)), tiles_k = tiles_of(total_k, 1, B, kSeqBwdKeys);
    MA_TRY(check_grid(std::max(tiles_q, tiles_k), Hkv));
    if ((total == 0 && total_k == 0) || (B == 0 && !clear)) return MA_OK;
    if (rest && dtype == MA_F32) return fail(MA_EINVAL, "rest is of 16-bit outputs");
    const size_t qb = span_bytes(total, Hq * d, Hq * d, dtype), kb = span_bytes(total_k, Hkv * d, Hkv * d, dtype), starts = (size_t)(B + 1) * 4;
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k", k, span_bytes(total_k, ldk, Hkv * d, dtype)},
                         {"v", v, span_bytes(total_k, ldv, Hkv * d, dtype)},
                         {"out", out, qb},
                         {"dout", dout, qb},
                         {"lse", lse, (size_t)(Hq * total) * 4},
                         {"cu_q", cu_q, starts},
                         {"cu_k", cu_k, starts},
                         {"k_lens", k_lens, k_lens ? (size_t)B * 4 : 0},
                         {"rest", rest, rest ? qb : 0}};
    const Range outs[] = {{"dq", dq, qb}, {"dk", dk, kb}, {"dv", dv, kb}};
    MA_TRY(check_ranges(ins, {16, 16, 16, 16, 16, 4, 4, 4, 4, 16}));
    MA_TRY(check_ranges(outs, {16, 16, 16}));
    MA_TRY(check_overlaps(outs, ins));
    CallScope c;
    MA_TRY(begin_call(c));
    const CrossPieces pieces = cross_pieces(B, total, total_k, tiles_q, tiles_k, Hkv, G, c.num_cus);
    const size_t part = pieces.keys > 1 ? (size_t)(pieces.keys * total_k * Hkv) * tile_d(d) * 4 : 0;
    const size_t part_q = pieces.rows > 1 ? (size_t)(pieces.rows * total * Hq) * tile_d(d) * 4 : 0;
    const size_t each = stat_bytes_of(total, Hq), norms = dtype == MA_F16 ? each + stat_bytes_of(total_k, Hkv) : 0;
    const size_t stat_bytes = 2 * each + norms;
    MA_TRY(check_grid(tiles_k * pieces.keys + tiles_q * pieces.rows, Hkv));
    MA_TRY(call_workspace(stream, stat_bytes + 2 * part + part_q, c));
    BwdLaunch x{};
    ma::SeqBwd &p = x.p;
    p.q = q, p.k = k, p.v = v, p.out = out, p.dout = dout, p.lse = lse, p.rest = rest;
    p.dq = dq, p.dk = dk, p.dv = dv;
    p.seqs = ma::Seqs{cu_q, (int)B, (int)total};
    p.keys = ma::KeySeqs{{cu_k, (int)B, (int)total_k}, k_lens};
    p.Hkv = (int)Hkv, p.G = (int)G, p.d = (int)d;
    p.ldq = ldq, p.ldk = ldk, p.ldv = ldv;
    p.c = log2_scale(d), p.clear = clear != 0;
    p.tiles_q = (int)tiles_q, p.tiles_k = (int)tiles_k;
    p.lse2 = (float *)c.ws, p.delta = (float *)(c.ws + each);
    if (dtype == MA_F16) p.norm_g = (float *)(c.ws + 2 * each), p.norm_v = (float *)(c.ws + 3 * each);
    p.stat_blocks = (int)std::max<int64_t>(1, std::min<int64_t>(kStatBlocks, (std::max(total * G, total_k) + 15) / 16 * Hkv));
    p.pieces = (int)pieces.keys, p.pieces_q = (int)pieces.rows;
    p.part_q = (float *)(c.ws + stat_bytes + 2 * part);
    p.part_k = (float *)(c.ws + stat_bytes), p.part_v = (float *)(c.ws + stat_bytes + part);
    x.dtype = dtype;
    return run_launches(stream, BwdLaunch::run, &x);
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
    const size_t cache = cache_bytes(pages, Hkv, page, d, dtype);
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

int monarch_attn_exact_cross_fwd(const void *q, const void *k, const void *v, void *out, float *lse, void *rest,
                                 const int32_t *cu_q, const int32_t *cu_k, const int32_t *k_lens, int64_t B, int64_t total,
                                 int64_t total_k, int64_t Hq, int64_t Hkv, int64_t d, int64_t ldq, int64_t ldk, int64_t ldv,
                                 int32_t clear, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return cross_fwd(q, k, v, out, lse, rest, cu_q, cu_k, k_lens, B, total, total_k, Hq, Hkv, d, ldq, ldk, ldv, clear, dtype,
                         (hipStream_t)stream);
    });
}

int monarch_attn_exact_cross_bwd(const void *q, const void *k, const void *v, const void *out, const float *lse, const void *rest,
                                 const void *dout, void *dq, void *dk, void *dv, const int32_t *cu_q, const int32_t *cu_k,
                                 const int32_t *k_lens, int64_t B, int64_t total, int64_t total_k, int64_t Hq, int64_t Hkv,
                                 int64_t d, int64_t ldq, int64_t ldk, int64_t ldv, int32_t clear, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return cross_bwd(q, k, v, out, lse, rest, dout, dq, dk, dv, cu_q, cu_k, k_lens, B, total, total_k, Hq, Hkv, d, ldq, ldk, ldv,
                         clear, dtype, (hipStream_t)stream);
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
