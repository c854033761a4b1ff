// Driver of the host code of the exact attention over sequences and of the
// paged cache (seq_abi.hip and what it shares of monarch_attn.hip) under
// AddressSanitizer and UndefinedBehaviorSanitizer.  The dispatch units are
// stand-ins; every call fails, or finishes, before any HIP call.
#include <cstdint>
#include <cstdio>

#include "../../paper_2505_18698_amd/csrc/seq_host.hpp"

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
    char *O = F + (uintptr_t(1) << 30);
    const int32_t *I = reinterpret_cast<const int32_t *>(F);
    float *L = reinterpret_cast<float *>(O);
    const int64_t big = INT64_MAX;
    auto fwd = [&](int64_t B, int64_t total, int64_t Hq, int64_t Hkv, int64_t d, int64_t ld, int32_t dtype) {
        return monarch_attn_exact_packed_fwd(F, F, F, O, nullptr, nullptr, I, B, total, Hq, Hkv, d, ld, ld, ld, 1, 0, dtype, nullptr);
    };
    expect(fwd(-1, 8, 4, 2, 64, 256, 1), MA_EINVAL, "B < 0");
    expect(fwd(1, 8, 4, 3, 64, 256, 1), MA_EINVAL, "Hq not a multiple of Hkv");
    expect(fwd(1, 8, 4, 2, 64, 250, 1), MA_EINVAL, "stride");
    expect(fwd(1, big, 4, 2, 64, 256, 1), MA_EUNSUPPORTED, "total beyond int64 products");
    expect(fwd(big, 8, 4, 2, 64, 256, 1), MA_EUNSUPPORTED, "B beyond int64 products");
    expect(fwd(1, 8, big, 1, 64, 256, 1), MA_EUNSUPPORTED, "Hq beyond int64 products");
    expect(fwd(1, 8, big, big, 64, 256, 1), MA_EUNSUPPORTED, "Hkv beyond int64 products");
    expect(fwd(1, 8, 4, 2, big, 256, 1), MA_EUNSUPPORTED, "d");
    expect(fwd(1, 8, 4, 2, 64, big, 1), MA_EINVAL, "stride beyond int64 products");
    expect(fwd(1, 8, 4, 2, 64, INT64_MIN, 1), MA_EINVAL, "negative stride");
    expect(fwd(0, 8, 4, 2, 64, 256, 1), MA_OK, "no sequence");
    expect(fwd(1, 0, 4, 2, 64, 256, 0), MA_OK, "no row");
    expect(fwd(1, 8, 4, 2, 64, 256, 5), MA_EINVAL, "dtype");
    expect(monarch_attn_exact_packed_fwd(F, F, F, F + 64, nullptr, nullptr, I, 1, 8, 4, 2, 64, 256, 256, 256, 1, 0, 1, nullptr), MA_EINVAL,
           "out overlaps q");
    expect(monarch_attn_exact_packed_bwd(F, F, F, F, L, nullptr, F, O, O, O, I, 1, 8, 4, 2, 64, 256, 256, 256, 1, 0, 1, nullptr), MA_EINVAL,
           "gradients overlap");
    expect(monarch_attn_exact_packed_bwd(nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr, nullptr,
                                         nullptr, 0, 0, 4, 2, 64, 256, 256, 256, 1, 0, 1, nullptr),
           MA_OK, "empty gradient");
    auto paged = [&](int64_t pages, int64_t page, int64_t blocks, int64_t B) {
        return monarch_attn_exact_paged_fwd(F, F, F, F, nullptr, I, I, I, B, 8, 4, 2, 64, 256, pages, page, blocks, 1, 1, nullptr);
    };
    expect(paged(4, 24, 4, 1), MA_EUNSUPPORTED, "page");
    expect(paged(big, 16, 4, 1), MA_EINVAL, "pages");
    expect(paged(4, 16, big, 1), MA_EINVAL, "blocks");
    expect(paged(4, 16, 4, 1), MA_EINVAL, "out overlaps q");
    expect(paged(4, 16, 4, 0), MA_OK, "no sequence");
    int32_t *W = reinterpret_cast<int32_t *>(O);
    int64_t *S = reinterpret_cast<int64_t *>(O);
    expect(monarch_attn_paged_plan(I, I, I, I, W, W, W, S, W, W, 2, 4, 4, 16, 8, nullptr), MA_EINVAL, "plan outputs overlap");
    expect(monarch_attn_paged_plan(I, I, I, I, W, W, W, S, W, W, big, 4, 4, 16, 8, nullptr), MA_EUNSUPPORTED, "plan B");
    expect(monarch_attn_paged_plan(I, I, I, I, W, W, W, S, W, W, 2, 4, 4, 17, 8, nullptr), MA_EUNSUPPORTED, "plan page");
    expect(monarch_attn_paged_write(F, F, F, F, S, 8, 2, 64, 128, 128, 4, 16, 1, nullptr), MA_EINVAL, "write over its input");
    expect(monarch_attn_paged_write(F, F, F, F, S, big, 2, 64, 128, 128, 4, 16, 1, nullptr), MA_EUNSUPPORTED, "write rows");
    expect(monarch_attn_paged_write(F, F, F, F, S, 0, 2, 64, 128, 128, 4, 16, 1, nullptr), MA_OK, "write nothing");
    if (fails == 0) std::printf("ok\n");
    return fails != 0;
}
