// Driver of the host code of cross attention and of a decoder's operators
// (seq_abi.hip, decoder_abi.hip and what they share of monarch_attn.hip) under
// AddressSanitizer and UndefinedBehaviorSanitizer.  The dispatch units are
// stand-ins; every call fails, or finishes, before any HIP call.
#include <cstdint>
#include <cstdio>

#include "../../paper_2505_18698_amd/csrc/decoder_host.hpp"

namespace ma_host {
#define MA_STANDIN(T)                                                                                          \
    template <> int run_call<T>(Launcher &, const CallBufs &, const CallDims &, int) { return MA_EHIP; }       \
    template <> int run_exact<T>(Launcher &, const CallBufs &, float *, int64_t, int, int) { return MA_EHIP; } \
    template <> int run_bwd<T>(Launcher &, const BwdCallBufs &, const CallDims &) { return MA_EHIP; }          \
    template <> int run_seq_fwd<T>(Launcher &, const ma::SeqFwd &, const SeqPlan &) { return MA_EHIP; }        \
    template <> int run_seq_bwd<T>(Launcher &, const ma::SeqBwd &) { return MA_EHIP; }
MA_STANDIN(float)
MA_STANDIN(__bf16)
MA_STANDIN(_Float16)
int run_paged_plan(Launcher &, const ma::PagedPlan &) { return MA_EHIP; }
int run_paged_write(Launcher &, const ma::PagedWrite &) { return MA_EHIP; }
int run_rotate(Launcher &, const ma::Rotate &, int32_t, bool) { return MA_EHIP; }
int run_beam_select(Launcher &, const ma::BeamSelect &, int32_t) { return MA_EHIP; }
int run_paged_reorder(Launcher &, const ma::PagedReorder &) { return MA_EHIP; }
}  // namespace ma_host

static int fails = 0;

static void expect(int got, int want, const char *what)
{
    if (got != want) {
        std::fprintf(stderr, "FAILED: %s: %d (%s)\n", what, got, monarch_attn_last_error());
        ++fails;
    }
}

int main()
{
    char *F = reinterpret_cast<char *>(uintptr_t(1) << 20);  // aligned, never dereferenced
    char *O = F + (uintptr_t(1) << 40);
    const int32_t *I = reinterpret_cast<const int32_t *>(F);
    const float *X = reinterpret_cast<const float *>(F);
    float *L = reinterpret_cast<float *>(O);
    int32_t *W = reinterpret_cast<int32_t *>(O);
    const int64_t *S = reinterpret_cast<const int64_t *>(F);
    const uint8_t *D = reinterpret_cast<const uint8_t *>(F);
    const int64_t big = INT64_MAX, low = INT64_MIN;

    auto cross = [&](int64_t B, int64_t total, int64_t total_k, int64_t Hq, int64_t Hkv, int64_t d, int64_t ld) {
        return monarch_attn_exact_cross_fwd(F, F, F, F, nullptr, nullptr, I, I, I, B, total, total_k, Hq, Hkv, d, ld, ld, ld, 0, 1, nullptr);
    };
    expect(cross(1, 8, 8, 4, 2, 64, 256), MA_EINVAL, "cross: out overlaps q");
    expect(cross(big, 8, 8, 4, 2, 64, 256), MA_EUNSUPPORTED, "cross: B");
    expect(cross(1, big, 8, 4, 2, 64, 256), MA_EUNSUPPORTED, "cross: total");
    expect(cross(1, 8, big, 4, 2, 64, 256), MA_EUNSUPPORTED, "cross: total_k");
    expect(cross(1, 8, low, 4, 2, 64, 256), MA_EINVAL, "cross: total_k < 0");
    expect(cross(1, 8, 8, big, 1, 64, 256), MA_EUNSUPPORTED, "cross: Hq");
    expect(cross(1, 8, 8, 4, 2, big, 256), MA_EUNSUPPORTED, "cross: d");
    expect(cross(1, 8, 8, 4, 2, 64, low), MA_EINVAL, "cross: stride");
    expect(cross(0, 8, 8, 4, 2, 64, 256), MA_OK, "cross: no sequence");
    // the largest sizes that pass the checks of sizes: their ranges overlap
    expect(cross(1 << 20, 1 << 24, 0x7fffff00, 4, 2, 64, 1 << 20), MA_EINVAL, "cross: large");
    auto grad = [&](int64_t B, int64_t total, int64_t total_k, int64_t Hq, int64_t Hkv) {
        return monarch_attn_exact_cross_bwd(F, F, F, F, X, nullptr, F, O, O, O, I, I, nullptr, B, total, total_k, Hq, Hkv, 64, 1 << 20, 1 << 20,
                                            1 << 20, 0, 1, nullptr);
    };
    expect(grad(1, 8, 8, 4, 2), MA_EINVAL, "cross: gradients overlap");
    expect(grad(1, 8, big, 4, 2), MA_EUNSUPPORTED, "cross gradient: total_k");
    expect(grad(1 << 20, 1 << 24, 1 << 26, 4, 2), MA_EINVAL, "cross gradient: large");
    expect(grad(1, 0, 0, 4, 2), MA_OK, "cross gradient: nothing");

    auto rotate = [&](int64_t B, int64_t total, int64_t Hq, int64_t Hk, int64_t d, int64_t rot, int64_t ld) {
        return monarch_attn_rotate(F, F, F, O, X, I, I, B, total, Hq, Hk, d, rot, ld, ld, 0, 0, 0, 1, nullptr);
    };
    expect(rotate(1, 8, 4, 2, 64, 64, 256), MA_EINVAL, "rotate: q_out overlaps q");
    expect(rotate(big, 8, 4, 2, 64, 64, 256), MA_EUNSUPPORTED, "rotate: B");
    expect(rotate(1, big, 4, 2, 64, 64, 256), MA_EUNSUPPORTED, "rotate: total");
    expect(rotate(1, 8, big, 2, 64, 64, 256), MA_EUNSUPPORTED, "rotate: Hq");
    expect(rotate(1, 8, 4, big, 64, 64, 256), MA_EUNSUPPORTED, "rotate: Hk");
    expect(rotate(1, 8, 4, low, 64, 64, 256), MA_EINVAL, "rotate: Hk < 0");
    expect(rotate(1, 8, 4, 2, big, 64, 256), MA_EUNSUPPORTED, "rotate: d");
    expect(rotate(1, 8, 4, 2, 64, big, 256), MA_EINVAL, "rotate: rot");
    expect(rotate(1, 8, 4, 2, 64, low, 256), MA_EINVAL, "rotate: rot < 0");
    expect(rotate(1, 8, 4, 2, 64, 64, big), MA_EINVAL, "rotate: stride");
    expect(rotate(1, 0, 4, 2, 64, 64, 256), MA_OK, "rotate: no row");
    expect(rotate(1, 1 << 17, 1 << 13, 1 << 13, 64, 64, 1 << 20), MA_EINVAL, "rotate: large");

    auto append = [&](int64_t total, int64_t Hkv, int64_t ldv, int64_t pages, int64_t page) {
        return monarch_attn_paged_append(F, F, F, F, O, O, X, I, I, S, 1, total, 4, Hkv, 64, 64, 256, 256, ldv, pages, page, 0, 1, nullptr);
    };
    expect(append(8, 2, 256, 4, 16), MA_EINVAL, "append: q_out overlaps q");
    expect(append(8, low, 256, 4, 16), MA_EINVAL, "append: Hkv < 0");
    expect(append(8, 0, 256, 4, 16), MA_EINVAL, "append: Hkv 0");
    expect(append(8, 2, big, 4, 16), MA_EINVAL, "append: stride");
    expect(append(8, 2, 256, big, 16), MA_EINVAL, "append: pages");
    expect(append(8, 2, 256, 4, big), MA_EUNSUPPORTED, "append: page");
    expect(append(8, 2, 256, 0x7fffffff, 4096), MA_EINVAL, "append: a large cache");
    expect(append(0, 2, 256, 4, 16), MA_OK, "append: no row");

    auto select = [&](int64_t B, int64_t K, int64_t V, int64_t M, int64_t ld, int32_t eos, int32_t dtype) {
        return monarch_attn_beam_select(F, X, D, reinterpret_cast<float *>(F), W, W, nullptr, B, K, V, M, ld, eos, dtype, nullptr);
    };
    expect(select(1, 4, 100, 8, 100, 2, 1), MA_EINVAL, "select: scores_out overlaps logits");
    expect(select(big, 4, 100, 8, 100, 2, 1), MA_EUNSUPPORTED, "select: B");
    expect(select(0x7fffffff, 32, 524288, 32, 524288, 2, 0), MA_EUNSUPPORTED, "select: parts");
    expect(select(1, big, 100, 8, 100, 2, 1), MA_EUNSUPPORTED, "select: K");
    expect(select(1, 4, big, 8, big, 2, 1), MA_EUNSUPPORTED, "select: V");
    expect(select(1, 4, 100, big, 100, 2, 1), MA_EUNSUPPORTED, "select: M");
    expect(select(1, 4, 100, 8, big, 2, 1), MA_EUNSUPPORTED, "select: ld");
    expect(select(1, 4, 100, 8, low, 2, 1), MA_EINVAL, "select: ld < 0");
    expect(select(1, 4, 100, 8, 100, INT32_MIN, 1), MA_EINVAL, "select: eos");
    expect(select(1, 4, 100, 8, 100, 2, 7), MA_EINVAL, "select: dtype");
    expect(select(low, 4, 100, 8, 100, 2, 1), MA_EINVAL, "select: B < 0");
    expect(select(0, 4, 100, 8, 100, 2, 1), MA_OK, "select: no request");
    expect(select(1 << 14, 32, 524288, 32, int64_t(1) << 31, 2, 0), MA_EINVAL, "select: large");

    auto reorder = [&](int64_t B, int64_t K, int64_t Hkv, int64_t pages, int64_t page, int64_t blocks) {
        return monarch_attn_paged_reorder(O, O, W, I, I, B, K, Hkv, 64, pages, page, blocks, 1, 1, nullptr);
    };
    expect(reorder(2, 4, 2, 4, 16, 4), MA_EINVAL, "reorder: pages overlap");
    expect(reorder(big, 4, 2, 4, 16, 4), MA_EUNSUPPORTED, "reorder: B");
    expect(reorder(2, big, 2, 4, 16, 4), MA_EUNSUPPORTED, "reorder: K");
    expect(reorder(2, 4, big, 4, 16, 4), MA_EUNSUPPORTED, "reorder: Hkv");
    expect(reorder(2, 4, 2, big, 16, 4), MA_EINVAL, "reorder: pages");
    expect(reorder(2, 4, 2, 4, low, 4), MA_EUNSUPPORTED, "reorder: page");
    expect(reorder(2, 4, 2, 4, 16, big), MA_EINVAL, "reorder: blocks");
    expect(reorder(65535, 32, 1 << 14, 0x7fffffff, 4096, 0x7fffffff), MA_EINVAL, "reorder: large");
    expect(reorder(0, 4, 2, 4, 16, 4), MA_OK, "reorder: no request");
    if (fails == 0) std::printf("ok\n");
    return fails != 0;
}
