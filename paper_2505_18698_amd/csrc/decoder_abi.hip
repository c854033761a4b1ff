// C ABI of a decoder's rotation, beams and cache order (include/monarch_attn.h): argument checks,
// workspaces and how a call runs.
#include <algorithm>

#include "decoder_host.hpp"
#include "seq_checks.hpp"

namespace {

using namespace ma_host;

struct RotateLaunch {
    ma::Rotate p;
    int32_t dtype;
    bool append;
    static int run(Launcher &L, void *a)
    {
        const RotateLaunch &x = *(const RotateLaunch *)a;
        return run_rotate(L, x.p, x.dtype, x.append);
    }
};

int check_rotation(int64_t B, int64_t total, int64_t Hq, int64_t Hk, int64_t d, int64_t rot, int64_t ldq, int64_t ldk, int32_t dtype)
{
    MA_TRY(check_heads(B, total, Hq, 1, d, dtype));
    if (Hk < 0) return fail(MA_EINVAL, "the heads of k must be >= 0");
    if (Hk > 0) MA_TRY(check_heads(B, total, Hk, 1, d, dtype));
    if (rot < 2 || rot > d || rot % 2) return fail(MA_EINVAL, "rot must be even and in 2..d (got %lld)", (long long)rot);
    if (rot % 8) return fail(MA_EUNSUPPORTED, "rot must be a multiple of 8 (got %lld)", (long long)rot);
    MA_TRY(check_stride("ldq", ldq, Hq * d, dtype));
    return Hk > 0 ? check_stride("ldk", ldk, Hk * d, dtype) : MA_OK;
}

// Rows a workgroup takes: as many as keep its threads busy a few times, as long as two workgroups a
// compute unit are left.
int rotate_rows(int64_t total, int64_t heads, int64_t d, int32_t dtype)
{
    const int64_t items = heads * ((d * (int64_t)elem_bytes(dtype) + 31) / 32);
    return (int)std::max<int64_t>(1, std::min<int64_t>({ma::kRotateRows, 1536 / items, total / 512}));
}

int rotate(const void *q, const void *k, void *q_out, void *k_out, const float *inv_freq, const int32_t *cu, const int32_t *kv_lens,
           int64_t B, int64_t total, int64_t Hq, int64_t Hk, int64_t d, int64_t rot, int64_t ldq, int64_t ldk, int32_t interleaved,
           int32_t inverse, int32_t clear, int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_rotation(B, total, Hq, Hk, d, rot, ldq, ldk, dtype));
    const int rows = rotate_rows(total, Hq + Hk, d, dtype);
    MA_TRY(check_grid((total + rows - 1) / rows, 1));
    if (total == 0 || (B == 0 && !clear)) return MA_OK;
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k", Hk ? k : nullptr, Hk ? span_bytes(total, ldk, Hk * d, dtype) : 0},
                         {"inv_freq", inv_freq, (size_t)rot / 2 * 4},
                         {"cu_seqlens", cu, (size_t)(B + 1) * 4},
                         {"kv_lens", kv_lens, kv_lens ? (size_t)B * 4 : 0}};
    const Range outs[] = {{"q_out", q_out, span_bytes(total, Hq * d, Hq * d, dtype)},
                          {"k_out", Hk ? k_out : nullptr, Hk ? span_bytes(total, Hk * d, Hk * d, dtype) : 0}};
    MA_TRY(check_ranges(ins, {16, 16, 4, 4, 4}));
    MA_TRY(check_ranges(outs, {16, 16}));
    MA_TRY(check_overlaps(outs, ins));
    RotateLaunch x{};
    ma::Rotate &p = x.p;
    p.q = q, p.k = k, p.q_out = q_out, p.k_out = k_out, p.inv_freq = inv_freq;
    p.seqs = ma::Seqs{cu, (int)B, (int)total}, p.kv_lens = kv_lens;
    p.Hq = (int)Hq, p.Hk = (int)Hk, p.d = (int)d, p.rot = (int)rot, p.ldq = ldq, p.ldk = ldk;
    p.interleaved = interleaved != 0, p.inverse = inverse != 0, p.clear = clear != 0, p.rows = rows;
    x.dtype = dtype;
    return run_launches(stream, RotateLaunch::run, &x);
}

int append(const void *q, const void *k, const void *v, void *q_out, void *k_pages, void *v_pages, const float *inv_freq,
           const int32_t *cu, const int32_t *kv_lens, const int64_t *slots, int64_t B, int64_t total, int64_t Hq, int64_t Hkv,
           int64_t d, int64_t rot, int64_t ldq, int64_t ldk, int64_t ldv, int64_t pages, int64_t page, int32_t interleaved,
           int32_t dtype, hipStream_t stream)
{
    MA_TRY(check_rotation(B, total, Hq, Hkv, d, rot, ldq, ldk, dtype));
    if (Hkv < 1) return fail(MA_EINVAL, "Hkv must be >= 1");
    MA_TRY(check_stride("ldv", ldv, Hkv * d, dtype));
    MA_TRY(check_pages(pages, page));
    const int rows = rotate_rows(total, Hq + 2 * Hkv, d, dtype);
    MA_TRY(check_grid((total + rows - 1) / rows, 1));
    if (total == 0 || B == 0) return MA_OK;
    const size_t cache = cache_bytes(pages, Hkv, page, d, dtype);
    const Range ins[] = {{"q", q, span_bytes(total, ldq, Hq * d, dtype)},
                         {"k", k, span_bytes(total, ldk, Hkv * d, dtype)},
                         {"v", v, span_bytes(total, ldv, Hkv * d, dtype)},
                         {"inv_freq", inv_freq, (size_t)rot / 2 * 4},
                         {"cu_seqlens", cu, (size_t)(B + 1) * 4},
                         {"kv_lens", kv_lens, (size_t)B * 4},
                         {"slots", slots, (size_t)total * 8}};
    const Range outs[] = {{"q_out", q_out, span_bytes(total, Hq * d, Hq * d, dtype)}, {"k_pages", k_pages, cache}, {"v_pages", v_pages, cache}};
    MA_TRY(check_ranges(ins, {16, 16, 16, 4, 4, 4, 8}));
    MA_TRY(check_ranges(outs, {16, 16, 16}));
    MA_TRY(check_overlaps(outs, ins));
    RotateLaunch x{};
    ma::Rotate &p = x.p;
    p.q = q, p.k = k, p.v = v, p.q_out = q_out, p.k_out = k_pages, p.v_out = v_pages, p.inv_freq = inv_freq;
    p.seqs = ma::Seqs{cu, (int)B, (int)total}, p.kv_lens = kv_lens, p.slots = slots;
    p.Hq = (int)Hq, p.Hk = (int)Hkv, p.d = (int)d, p.rot = (int)rot, p.ldq = ldq, p.ldk = ldk, p.ldv = ldv;
    p.page_log2 = log2_of(page), p.pages = (int)pages;
    p.interleaved = interleaved != 0, p.rows = rows;
    x.dtype = dtype, x.append = true;
    return run_launches(stream, RotateLaunch::run, &x);
}

struct SelectLaunch {
    ma::BeamSelect p;
    int32_t dtype;
    static int run(Launcher &L, void *a)
    {
        const SelectLaunch &x = *(const SelectLaunch *)a;
        return run_beam_select(L, x.p, x.dtype);
    }
};

// How the rows are divided: as many parts as make four workgroups a compute unit, of 8192 tokens at
// least, and no more than 256 lists a request, or 8 a beam, for what is left to do in one workgroup. (64 requests of
// 8 beams over 50001 tokens in bf16, 16 taken: 26 us, 29 with half or twice as many workgroups. One
// request of 16 beams over 200000 in fp16, 32 taken: 33 us, 47 with 25 parts, 37 with 4.)
struct BeamParts {
    int64_t parts, vectors;  // of 16 bytes a part
};

BeamParts beam_parts(int64_t rows, int64_t K, int64_t V, int32_t dtype)
{
    const int64_t all = std::max<int64_t>(1, V * (int64_t)elem_bytes(dtype) / 16), most = (V + 8191) / 8192;
    const int64_t parts = std::max<int64_t>(1, std::min({most, (1024 + rows - 1) / std::max<int64_t>(1, rows), std::max<int64_t>(8, 256 / K)}));
    BeamParts how;
    how.vectors = (all + parts - 1) / parts;
    how.parts = (all + how.vectors - 1) / how.vectors;
    return how;
}

int select(const void *logits, const float *scores, const uint8_t *done, float *scores_out, int32_t *tokens, int32_t *parents,
           uint8_t *done_out, int64_t B, int64_t K, int64_t V, int64_t M, int64_t ld, int32_t eos, int32_t dtype, hipStream_t stream)
{
    if (dtype != MA_F32 && dtype != MA_BF16 && dtype != MA_F16) return fail(MA_EINVAL, "unknown dtype %d", dtype);
    if (B < 0 || K < 1 || V < 1 || M < 1) return fail(MA_EINVAL, "B must be >= 0, K, V and M >= 1");
    if (K > MONARCH_ATTN_BEAM_MAX || M > MONARCH_ATTN_BEAM_MAX)
        return fail(MA_EUNSUPPORTED, "K and M must not exceed %d", MONARCH_ATTN_BEAM_MAX);
    if (V > MONARCH_ATTN_BEAM_MAX_VOCAB) return fail(MA_EUNSUPPORTED, "V must not exceed %d", MONARCH_ATTN_BEAM_MAX_VOCAB);
    if (M > K * V) return fail(MA_EINVAL, "M (%lld) must not exceed K V (%lld)", (long long)M, (long long)(K * V));
    if (ld < V) return fail(MA_EINVAL, "ld (%lld) must be at least V", (long long)ld);
    if (ld > int64_t(1) << 31 || B > 0x7fffffff) return fail(MA_EUNSUPPORTED, "ld and B must not exceed 2^31");
    if ((done || done_out) && (eos < 0 || eos >= V)) return fail(MA_EINVAL, "eos must be a token with done or done_out");
    const BeamParts how = beam_parts(B * K, K, V, dtype);
    const int64_t parts = how.parts;
    MA_TRY(check_grid(B * K * parts, 1));
    if (B == 0) return MA_OK;
    const size_t beams = (size_t)(B * K), out = (size_t)(B * M);
    const Range ins[] = {{"logits", logits, span_bytes(B * K, ld, V, dtype)},
                         {"scores", scores, beams * 4},
                         {"done", done, done ? beams : 0}};
    const Range outs[] = {{"scores_out", scores_out, out * 4}, {"tokens", tokens, out * 4}, {"parents", parents, out * 4},
                          {"done_out", done_out, done_out ? out : 0}};
    MA_TRY(check_ranges(ins, {elem_bytes(dtype), 4, 1}));
    MA_TRY(check_ranges(outs, {4, 4, 4, 1}));
    MA_TRY(check_overlaps(outs, ins));
    CallScope c;
    MA_TRY(begin_call(c));
    const size_t all = beams * parts, keys = align_up(all * M * 8), stats = align_up(all * 4);
    MA_TRY(call_workspace(stream, keys + 2 * stats, c));
    SelectLaunch x{};
    ma::BeamSelect &p = x.p;
    p.logits = logits, p.scores = scores, p.done = done;
    p.scores_out = scores_out, p.tokens = tokens, p.parents = parents, p.done_out = done_out;
    p.ld = ld, p.B = (int)B, p.K = (int)K, p.V = (int)V, p.M = (int)M, p.eos = eos;
    p.parts = (int)parts, p.part_vectors = (int)how.vectors;
    p.keys = (uint64_t *)c.ws, p.part_max = (float *)(c.ws + keys), p.part_sum = (float *)(c.ws + keys + stats);
    x.dtype = dtype;
    return run_launches(stream, SelectLaunch::run, &x);
}

int reorder(void *k_pages, void *v_pages, int32_t *table, const int32_t *parents, const int32_t *lens, int64_t B, int64_t K,
            int64_t Hkv, int64_t d, int64_t pages, int64_t page, int64_t blocks, int32_t move_table, int32_t dtype, hipStream_t stream)
{
    if (K < 1) return fail(MA_EINVAL, "K must be >= 1");
    if (K > MONARCH_ATTN_BEAM_MAX) return fail(MA_EUNSUPPORTED, "K must not exceed %d", MONARCH_ATTN_BEAM_MAX);
    if (B < 0) return fail(MA_EINVAL, "B must be >= 0");
    if (B > 65535) return fail(MA_EUNSUPPORTED, "B must not exceed 65535");
    MA_TRY(check_heads(B, B * K, Hkv, Hkv, d, dtype));
    MA_TRY(check_pages(pages, page));
    if (blocks < 0 || blocks > 0x7fffffff) return fail(MA_EINVAL, "blocks must be in 0..2^31 - 1");
    if (B == 0 || K == 1 || blocks == 0) return MA_OK;  // (a beam alone is its own parent)
    const size_t cache = cache_bytes(pages, Hkv, page, d, dtype);
    const Range ins[] = {{"parents", parents, (size_t)(B * K) * 4}, {"lens", lens, (size_t)(B * K) * 4}};
    const Range outs[] = {{"k_pages", k_pages, cache}, {"v_pages", v_pages, cache}, {"block_table", table, (size_t)(B * K * blocks) * 4}};
    MA_TRY(check_ranges(ins, {4, 4}));
    MA_TRY(check_ranges(outs, {16, 16, 4}));
    MA_TRY(check_overlaps(outs, ins));
    ma::PagedReorder p{k_pages, v_pages, table, parents, lens, (int)B, (int)K, (int)(d * elem_bytes(dtype) / 16), (int)Hkv,
                       log2_of(page), (int)pages, (int)blocks, move_table != 0};
    return run_launches(stream, [](Launcher &L, void *a) { return run_paged_reorder(L, *(const ma::PagedReorder *)a); }, &p);
}

}  // namespace

extern "C" {

int monarch_attn_rotate(const void *q, const void *k, void *q_out, void *k_out, const float *inv_freq, const int32_t *cu_seqlens,
                        const int32_t *kv_lens, int64_t B, int64_t total, int64_t Hq, int64_t Hk, int64_t d, int64_t rot,
                        int64_t ldq, int64_t ldk, int32_t interleaved, int32_t inverse, int32_t clear, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return rotate(q, k, q_out, k_out, inv_freq, cu_seqlens, kv_lens, B, total, Hq, Hk, d, rot, ldq, ldk, interleaved, inverse, clear,
                      dtype, (hipStream_t)stream);
    });
}

int monarch_attn_paged_append(const void *q, const void *k, const void *v, void *q_out, void *k_pages, void *v_pages,
                              const float *inv_freq, const int32_t *cu_seqlens, const int32_t *kv_lens, const int64_t *slots,
                              int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int64_t rot, int64_t ldq, int64_t ldk,
                              int64_t ldv, int64_t pages, int64_t page, int32_t interleaved, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return append(q, k, v, q_out, k_pages, v_pages, inv_freq, cu_seqlens, kv_lens, slots, B, total, Hq, Hkv, d, rot, ldq, ldk, ldv,
                      pages, page, interleaved, dtype, (hipStream_t)stream);
    });
}

int monarch_attn_beam_select(const void *logits, const float *scores, const uint8_t *done, float *scores_out, int32_t *tokens,
                             int32_t *parents, uint8_t *done_out, int64_t B, int64_t K, int64_t V, int64_t M, int64_t ld, int32_t eos,
                             int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return select(logits, scores, done, scores_out, tokens, parents, done_out, B, K, V, M, ld, eos, dtype, (hipStream_t)stream);
    });
}

int monarch_attn_paged_reorder(void *k_pages, void *v_pages, int32_t *block_table, const int32_t *parents, const int32_t *lens,
                               int64_t B, int64_t K, int64_t Hkv, int64_t d, int64_t pages, int64_t page, int64_t blocks,
                               int32_t move_table, int32_t dtype, void *stream)
{
    g_err[0] = '\0';
    return guarded([&] {
        return reorder(k_pages, v_pages, block_table, parents, lens, B, K, Hkv, d, pages, page, blocks, move_table, dtype,
                       (hipStream_t)stream);
    });
}

}  // extern "C"
