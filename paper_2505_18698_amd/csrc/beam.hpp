// Selection of the best continuations of a request's beams, and the paged cache in the order of the
// beams chosen.
//
// Candidate (k, t): beam k of score s_k goes on with token t, of logit x_kt:
//   s_k + x_kt - log sum_u exp(x_ku),
// a done beam only with the end token, at its own score.  The M largest of a request, in order, equal
// ones by the lowest (k, t).
#pragma once

#include "decoder_host.hpp"
#include "tiles.hpp"

namespace ma {

// A 32-bit integer in the order of the float (-0 as 0).
__device__ inline uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ inline float unordered(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
// The same of a double, in 64 bits.
__device__ inline uint64_t ordered(double x)
{
    const uint64_t u = (uint64_t)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ inline double unordered(uint64_t u) { return __longlong_as_double((int64_t)(u >> 63 ? u & ~(1ull << 63) : ~u)); }

// A logit and its token in the order of the candidates of a beam; 0 is behind all of them.
__device__ inline uint64_t key_of(float x, uint32_t token) { return (uint64_t)ordered(x) << 32 | (0xffffffffu - token); }

// Of the wave's values the largest one that at least m lanes reach (0 where fewer have one).
__device__ inline uint32_t reached_by(uint32_t x, int m)
{
    uint32_t t = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t with = t | 1u << bit;
        if (__popcll(__ballot(x >= with)) >= m) t = with;
    }
    return t;
}

// One part of a row a workgroup, held in registers: its largest logit, its sum of exponentials and
// its M best.  Of the lanes' best the M-th of a wave bounds the M-th of the part from below, and the
// largest such bound of the four waves is reached by few elements: those go to a list, in any order,
// and each finds its place by counting the larger ones.
template <typename T> __global__ __launch_bounds__(256) void beam_parts(BeamSelect p)
{
    constexpr int VE = 16 / (int)sizeof(T), NV = 32 / VE, E = NV * VE;
    // A wave's bound is reached by M lanes of it at most, with E elements each.
    __shared__ uint64_t list[4 * kBeamMax * E];
    __shared__ uint64_t bounds[4];
    __shared__ float maxima[4], sums[4];
    __shared__ int count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int part = blockIdx.x % p.parts;
    const int64_t row = blockIdx.x / p.parts;
    if (p.done && p.done[row]) return;
    if (p.scores[row] == -INFINITY) return;
    if (tid == 0) count = 0;
    const T *x0 = (const T *)p.logits + row * p.ld;
    // vectors lie at whole 16 bytes, whatever the row does; element e of vector v is token v VE - shift + e
    const int shift = (int)((uintptr_t)x0 % 16 / sizeof(T));
    float x[E];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t t0 = ((int64_t)(part * NV + i) * 256 + tid) * VE - shift;
        T y[VE];
        if (t0 >= 0 && t0 + VE <= p.V) {
            __builtin_memcpy(y, __builtin_assume_aligned(x0 + t0, 16), 16);
        } else {
#pragma unroll
            for (int e = 0; e < VE; ++e) y[e] = t0 + e >= 0 && t0 + e < p.V ? x0[t0 + e] : (T)-INFINITY;
        }
#pragma unroll
        for (int e = 0; e < VE; ++e) x[i * VE + e] = (float)y[e];
    }
    auto token = [&](int j) { return ((part * NV + j / VE) * 256 + tid) * VE - shift + j % VE; };

    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < E; ++j) most = max_nan(most, x[j]);
    const float base = fabsf(most) < INFINITY ? most : 0.f;
    float sum = 0.f;
#pragma unroll
    for (int j = 0; j < E; ++j) sum += __builtin_amdgcn_exp2f((x[j] - base) * kLog2e);
    uint64_t best = 0;
#pragma unroll
    for (int j = E - 1; j >= 0; --j)
        if (x[j] == most && (uint32_t)token(j) < (uint32_t)p.V) best = key_of(x[j], (uint32_t)token(j));

    // (a row of which a logit is NaN or +infinity has no candidates: its keys are not read)
    float wave_most = most;
    for (int s = 1; s < 64; s <<= 1) wave_most = max_nan(wave_most, __shfl_xor(wave_most, s));
    const float wave_base = fabsf(wave_most) < INFINITY ? wave_most : 0.f;
    sum *= most == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((base - wave_base) * kLog2e);
    for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
    uint64_t bound = (uint64_t)reached_by((uint32_t)(best >> 32), p.M) << 32;
    if (bound && __popcll(__ballot(best >= bound)) > p.M) {  // several lanes with the last one's logit: the lowest tokens
        const uint32_t hi = (uint32_t)(bound >> 32);
        const int above = __popcll(__ballot((uint32_t)(best >> 32) > hi));
        bound |= reached_by((uint32_t)(best >> 32) == hi ? (uint32_t)best : 0u, p.M - above);
    }
    if (lane == 0) bounds[wave] = bound, maxima[wave] = wave_most, sums[wave] = sum;
    __syncthreads();
    bound = max(max(max(bounds[0], bounds[1]), max(bounds[2], bounds[3])), (uint64_t)1);
    if (tid == 0) {
        float m = maxima[0], s = 0.f;
        for (int i = 1; i < 4; ++i) m = max_nan(m, maxima[i]);
        for (int i = 0; i < 4; ++i) s += sums[i] * (maxima[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((maxima[i] - m) * kLog2e));
        p.part_max[blockIdx.x] = m, p.part_sum[blockIdx.x] = s;
    }
    if (best >= bound) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const uint32_t t = (uint32_t)token(j);
            if (t < (uint32_t)p.V && key_of(x[j], t) >= bound) list[atomicAdd(&count, 1)] = key_of(x[j], t);
        }
    }
    __syncthreads();
    uint64_t *out = p.keys + (int64_t)blockIdx.x * p.M;
    const int n = count;
    for (int i = tid; i < n; i += 256) {
        const uint64_t mine = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > mine;
        if (rank < p.M) out[rank] = mine;
    }
    if (tid >= n && tid < p.M) out[tid] = 0;
}

// One request a workgroup: every beam's sum from its parts, in 64 bits, so that candidates of
// different beams that are close to each other come out in order; then the M best of the parts' lists, all of which are
// in order: only the lists of the M best first entries count, and of these the entries that reach
// the last of them.
struct BeamEntry {
    uint64_t value, at;  // ordered(candidate); ~(beam V + token), so that both are "more is first"
    __device__ inline bool operator>(const BeamEntry &o) const { return value > o.value || (value == o.value && at > o.at); }
};

static __global__ __launch_bounds__(256) void beam_join(BeamSelect p)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    BeamEntry *heads = reinterpret_cast<BeamEntry *>(lds);  // of the lists; one behind them: the bound
    __shared__ BeamEntry list[kBeamMax * kBeamMax];
    __shared__ double lse[kBeamMax];
    __shared__ int kind[kBeamMax];  // of a beam: 0 candidates by its logits, 1 done, 2 all of them -infinity
    __shared__ int open[kBeamMax];  // lists that count
    __shared__ int opened, count;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row0 = (int64_t)blockIdx.x * p.K;
    const int lists = p.K * p.parts;
    if (tid == 0) opened = 0, count = 0;
    for (int k = wave; k < p.K; k += 4) {
        const int64_t row = row0 + k;
        const float score = p.scores[row];
        const bool dead = !(score > -INFINITY), ended = p.done && p.done[row];
        float most = -INFINITY;
        double sum = 0.0;
        if (!dead && !ended) {
            for (int i = lane; i < p.parts; i += 64) most = max_nan(most, p.part_max[row * p.parts + i]);
            for (int s = 1; s < 64; s <<= 1) most = max_nan(most, __shfl_xor(most, s));
            if (fabsf(most) < INFINITY)
                for (int i = lane; i < p.parts; i += 64)
                    sum += (double)p.part_sum[row * p.parts + i] * exp((double)p.part_max[row * p.parts + i] - (double)most);
            for (int s = 1; s < 64; s <<= 1) sum += __shfl_xor(sum, s);
        }
        if (lane == 0) {
            kind[k] = dead ? 2 : ended ? 1 : fabsf(most) < INFINITY ? 0 : 2;
            lse[k] = (double)most + log(sum);
        }
    }
    __syncthreads();
    // entry i of a list, or one behind all others
    auto entry = [&](int l, int i) {
        const int k = l / p.parts, part = l - k * p.parts;
        const double score = p.scores[row0 + k];
        BeamEntry e{0, 0};
        if (kind[k] == 0) {
            const uint64_t key = p.keys[((row0 + k) * p.parts + part) * p.M + i];
            if (key == 0) return e;
            const double x = score + ((double)unordered((uint32_t)(key >> 32)) - lse[k]);
            e.value = ordered(x == x ? x : -INFINITY);
            e.at = ~((uint64_t)k * p.V + (0xffffffffu - (uint32_t)key));
        } else if (part == 0 && i < p.V) {
            const bool first = kind[k] == 1 && i == 0;  // done: the end token, then the others, in front of it and behind it
            const int t = kind[k] == 2 ? i : first ? p.eos : i - 1 < p.eos ? i - 1 : i;
            e.value = ordered(first ? score : -(double)INFINITY);
            e.at = ~((uint64_t)k * p.V + t);
        }
        return e;
    };
    for (int l = tid; l < lists; l += 256) heads[l] = entry(l, 0);
    if (tid == 0) heads[lists] = BeamEntry{0, 0};
    __syncthreads();
    for (int l = tid; l < lists; l += 256) {
        const BeamEntry mine = heads[l];
        if (mine.value == 0) continue;
        int rank = 0;
        for (int j = 0; j < lists; ++j) rank += heads[j] > mine;
        if (rank < p.M) open[atomicAdd(&opened, 1)] = l;
        if (rank == p.M - 1) heads[lists] = mine;
    }
    __syncthreads();
    const BeamEntry bound = heads[lists];
    for (int i = tid; i < opened * p.M; i += 256) {
        const BeamEntry e = entry(open[i / p.M], i % p.M);
        if (e.value != 0 && !(bound > e)) list[atomicAdd(&count, 1)] = e;
    }
    __syncthreads();
    const int n = count;
    for (int i = tid; i < n; i += 256) {
        const BeamEntry mine = list[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += list[j] > mine;
        if (rank >= p.M) continue;
        const uint64_t at = ~mine.at;
        const int k = (int)(at / (uint32_t)p.V), t = (int)(at % (uint32_t)p.V);
        const int64_t to = (int64_t)blockIdx.x * p.M + rank;
        p.scores_out[to] = (float)unordered(mine.value);
        p.tokens[to] = t, p.parents[to] = k;
        if (p.done_out) p.done_out[to] = (p.done && p.done[row0 + k]) || t == p.eos;
    }
}

// The rows of the started page of every beam, and the table's entries of its full pages, from its
// parent, in place: a thread holds the same 16 bytes (the same entry) of all beams of a request, and
// stores none before all are loaded.  So no other thread has a part in what it reads and writes, and
// no copy of the cache is needed.  Beams that are their own parent cost nothing.
template <int KMAX> __global__ __launch_bounds__(256) void paged_reorder(PagedReorder p, int page_blocks)
{
    const int b = blockIdx.y, tid = threadIdx.x;
    const int n = max(0, p.lens[(int64_t)b * p.K]), full = n >> p.page_log2, rest = n & ((1 << p.page_log2) - 1);
    const int64_t row0 = (int64_t)b * p.K;
    int from[KMAX];
#pragma unroll
    for (int c = 0; c < KMAX; ++c) {
        from[c] = c < p.K ? p.parents[row0 + c] : c;
        if ((unsigned)from[c] >= (unsigned)p.K) from[c] = c;
    }
    if ((int)blockIdx.x >= page_blocks) {
        for (int j = ((int)blockIdx.x - page_blocks) * 256 + tid; j < min(full, p.blocks); j += ((int)gridDim.x - page_blocks) * 256) {
            int e[KMAX];
#pragma unroll
            for (int c = 0; c < KMAX; ++c)
                if (from[c] != c) e[c] = p.table[(row0 + from[c]) * p.blocks + j];
#pragma unroll
            for (int c = 0; c < KMAX; ++c)
                if (from[c] != c) p.table[(row0 + c) * p.blocks + j] = e[c];
        }
        return;
    }
    if (rest == 0 || full >= p.blocks) return;
    const int row = rest * p.chunks, each = p.Hkv * row;  // chunks of a head's rows, and of all heads
    const int64_t page = (int64_t)(p.Hkv << p.page_log2) * p.chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < 2ll * each; i += (int64_t)page_blocks * 256) {
        const int at = (int)(i < each ? i : i - each), head = at / row;
        u32x4 *cache = (u32x4 *)(i < each ? p.k_pages : p.v_pages) + (((int64_t)head << p.page_log2) * p.chunks + at - head * row);
        u32x4 x[KMAX];
        bool ok[KMAX];
        int to[KMAX];
#pragma unroll
        for (int c = 0; c < KMAX; ++c) {
            ok[c] = from[c] != c;
            if (!ok[c]) continue;
            const int src = p.table[(row0 + from[c]) * p.blocks + full];
            to[c] = p.table[(row0 + c) * p.blocks + full];
            ok[c] = (unsigned)src < (unsigned)p.pages && (unsigned)to[c] < (unsigned)p.pages;
            if (ok[c]) x[c] = cache[src * page];
        }
#pragma unroll
        for (int c = 0; c < KMAX; ++c)
            if (ok[c]) cache[to[c] * page] = x[c];
    }
}

}  // namespace ma
