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

// Of the wave's values the m-th largest, but for its lower `LOW` bits (0 where fewer than m have one): at
// least m lanes reach it.
template <int LOW> __device__ inline uint32_t reached_by(uint32_t x, int m)
{
    uint32_t t = 0;
#pragma unroll
    for (int bit = 31; bit >= LOW; --bit) {
        const uint32_t with = t | 1u << bit;
        if (__popcll(__ballot(x >= with)) >= m) t = with;
    }
    return t;
}

// How many of the first n entries of a list in LDS are larger than `mine`: eight at a time, so that their
// reads wait for each other no more than once.  (Up to seven behind the n-th are read.)
template <typename E> __device__ inline int larger_ones(const E *list, int n, const E &mine)
{
    int rank = 0;
    for (int j = 0; j < n; j += 8) {
        E x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = list[j + u];
#pragma unroll
        for (int u = 0; u < 8; ++u) rank += j + u < n && x[u] > mine;
    }
    return rank;
}

// The sum over a wave, the same in all lanes.
template <typename F> __device__ inline float over_wave(float x, F &&f)
{
    for (int s = 1; s < 64; s <<= 1) x = f(x, __shfl_xor(x, s));
    return x;
}

// exp(x - base) of logits, base no less than x; 0 of -infinity, whatever base is.
__device__ inline float exp_behind(float x, float base) { return x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x - base) * kLog2e); }

// A part of a row a workgroup, in chunks of 8192 tokens that are held in registers while the next one
// arrives: its largest logit, its sum of exponentials and its M best, in order.
//
// What reaches a bound goes to a list, in any order, and each entry finds its place by counting the
// larger ones.  The first chunk's bound: of the lanes' largest logits, the M-th of a wave, of the four
// waves the largest.  Later on it is the M-th best so far (equal logits come too late), which few
// exceed.  Where the list is too short all the same (thousands of equal logits, or ascending ones), a search
// over keys finds a bound that few enough reach.
//
// What bounds it: about 12 vector instructions a token, of which the exponential takes four issues, beside 2
// bytes. 64 requests of 8 beams over 50001 tokens in bf16 (51 MB, 16 taken): 19.6 us, vector instructions
// issue in 45 % of the time; by events, 14 of 21 us are the pass over the logits, 3 the first chunk's
// candidates, 4 the later ones'. 128000 tokens: 34 us by events. 4 beams over 32000 in fp32: 6.6 us, latency.
// (Where 98 % of the tokens are masked with -1e9 or less, the whole call takes 28.4 us for 26.7.)
template <typename T> __global__ __launch_bounds__(256) void beam_parts(BeamSelect p)
{
    constexpr int E = 32, VE = 16 / (int)sizeof(T), NV = E / VE, kRoom = 1024, kMany = 256;
    constexpr float kNear = 0x1p20f;  // of a reference below it the rounding is a sixteenth at most
    __shared__ __attribute__((aligned(16))) uint64_t list[kRoom + 8], best[kBeamMax];
    __shared__ uint32_t bounds[4];
    __shared__ float maxima[4], sums[4];
    __shared__ int count, found[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int part = blockIdx.x % p.parts;
    const int64_t row = blockIdx.x / p.parts;
    if (p.done && p.done[row]) return;
    if (p.scores[row] == -INFINITY) return;
    const T *x0 = (const T *)p.logits + row * p.ld;
    // A row starts anywhere in 16 bytes.  Its whole vectors, 16 bytes each, start at token `head`; the few
    // tokens in front of them belong to the first chunk of the row, those behind to the last, one a thread.
    const int head = min(p.V, (int)((16 - (uintptr_t)x0 % 16) % 16 / sizeof(T)));
    const int vectors = (p.V - head) / VE, end = head + vectors * VE;
    const int first = part * p.part_vectors, behind = min(vectors, first + p.part_vectors);
    const int chunks = max(1, (behind - first + NV * 256 - 1) / (NV * 256));
    u32x4 raw[NV];
    int lone = -1;  // this thread's token in front of the vectors, or behind them
    T lone_x;
    auto fetch = [&](int chunk) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = first + (chunk * NV + i) * 256 + tid;
            T none[VE];
#pragma unroll
            for (int e = 0; e < VE; ++e) none[e] = (T)-INFINITY;
            __builtin_memcpy(&raw[i], none, 16);
            if (v < behind) raw[i] = *((const u32x4 *)(x0 + head) + v);
        }
        lone = -1, lone_x = (T)-INFINITY;
        if (part == 0 && chunk == 0 && tid < head) lone = tid;
        if (part == p.parts - 1 && chunk == chunks - 1 && tid >= 64 && end + tid - 64 < p.V) lone = end + tid - 64;
        if (lone >= 0) lone_x = x0[lone];
    };
    fetch(0);
    if (tid == 0) count = 0;
    // of this thread's elements: the largest (NaN stays), and the sum of exponentials relative to it
    float most = -INFINITY, sum = 0.f;
    int kept = 0, listed = 0;           // entries of the list that are the best so far, in order, and all
    float bound = -INFINITY;            // with kept = M: the logit of the last of them
#pragma unroll 1
    for (int chunk = 0; chunk < chunks; ++chunk) {
        float x[E];
        bool some[NV];  // of the wave's vectors
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            T y[VE];
            __builtin_memcpy(y, &raw[i], 16);
            some[i] = first + (chunk * NV + i) * 256 + wave * 64 < behind;
#pragma unroll
            for (int e = 0; e < VE; ++e) x[i * VE + e] = (float)y[e];
        }
        const float y = (float)lone_x;
        const int at_y = lone;
        if (chunk + 1 < chunks) fetch(chunk + 1);
        const int t0 = head + (first + chunk * NV * 256) * VE;       // the first token of the chunk's vectors
        const int from = part == 0 && chunk == 0 ? 0 : t0;           // of the chunk
        auto token = [&](int j) { return t0 + (j / VE * 256 + tid) * VE + j % VE; };

        float top = y, tops[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            tops[i] = x[i * VE];
#pragma unroll
            for (int e = 1; e < VE; ++e) tops[i] = max_nan(tops[i], x[i * VE + e]);
            top = max_nan(top, tops[i]);
        }
        const float now = max_nan(most, top), base = fabsf(now) < INFINITY ? now : 0.f;
        float a = 0.f, b = 0.f;
        auto add_up = [&](auto &&exp_of) {
            a = exp_of(y);
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (some[i])
#pragma unroll
                    for (int e = 0; e < VE; e += 2) a += exp_of(x[i * VE + e]), b += exp_of(x[i * VE + e + 1]);
        };
        // exp(x - base): one instruction in front of the exponential, from the reference in units of log 2, which is
        // rounded; what that took is put right behind the sum.  Of large ones it would be too much for an exponential
        // (all of a thread's tokens masked with -1e10: 2^440), and the largest have no such reference.
        if (__all(fabsf(base) < kNear)) {
            const float scaled = base * kLog2e;
            add_up([&](float z) { return __builtin_amdgcn_exp2f(__builtin_fmaf(z, kLog2e, -scaled)); });
            const float by = __builtin_amdgcn_exp2f(-__builtin_fmaf(base, kLog2e, -scaled));
            a *= by, b *= by;
        } else {
            add_up([&](float z) { return exp_behind(z, base); });
        }
        sum = sum * exp_behind(most, base) + (a + b);
        most = now;

        float low = -INFINITY;  // bound of the first chunk's candidates
        if (kept == 0) {
            const uint32_t mine = reached_by<12>(ordered(top), p.M);  // (11 bits behind the exponent are enough)
            if (lane == 0) bounds[wave] = mine;
            __syncthreads();
            low = unordered(max(max(max(bounds[0], bounds[1]), max(bounds[2], bounds[3])), ordered(-INFINITY)));
        }
        uint32_t hits = 0;
        bool lone_hits = false;
        if (kept < p.M) {
            lone_hits = at_y >= 0 && y >= low;
            if (!(top < low))
#pragma unroll
                for (int j = 0; j < E; ++j) hits |= x[j] >= low ? 1u << j : 0u;
        } else if (!(top <= bound)) {
            lone_hits = y > bound;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (tops[i] > bound)
#pragma unroll
                    for (int e = 0; e < VE; ++e) hits |= x[i * VE + e] > bound ? 1u << (i * VE + e) : 0u;
        }
        while (hits || lone_hits) {  // few: their logits are read again, for registers cannot be picked by number
            const int t = lone_hits ? at_y : token(__builtin_ctz(hits));
            if (!lone_hits) hits &= hits - 1;
            const bool mine = lone_hits || t < head + behind * VE;
            lone_hits = false;
            if (!mine) continue;
            const float z = (float)x0[t];
            // (-infinity: of the M first tokens of the chunk alone, which have enough where any is needed)
            if (z == -INFINITY && t - from >= p.M) continue;
            const int at = atomicAdd(&count, 1);
            if (at < kRoom) list[at] = key_of(z, (uint32_t)t);
        }
        __syncthreads();
        int n = count;
        __syncthreads();  // (all have read it before the next chunk adds to it)
        if (n > kRoom) {
            // a key that at least M, and no more than the room, reach: bit by bit, from all threads' counts of
            // the chunk, read again
            auto reach = [&](int i, uint64_t with) {  // (the last one is the lone token)
                int t = t0 + i * 256 + tid;
                if (i == E || t >= head + behind * VE) t = i == E ? at_y : -1;
                const float z = t >= 0 ? (float)x0[t] : NAN;
                const uint64_t mine = z == z && (kept == 0 || z > bound) ? key_of(z, (uint32_t)t) : 0;
                return mine >= with ? mine : 0;
            };
            uint64_t key = 0;
#pragma unroll 1
            for (int bit = 63; bit >= 0; --bit) {
                const uint64_t with = key | 1ull << bit;
                int c = 0;
#pragma unroll 4
                for (int i = 0; i <= E; ++i) c += reach(i, with) != 0;
                for (int s = 1; s < 64; s <<= 1) c += __shfl_xor(c, s);
                __syncthreads();
                if (lane == 0) found[wave] = c;
                __syncthreads();
                c = found[0] + found[1] + found[2] + found[3];
                if (c >= p.M) key = with;
                if (c >= p.M && c <= kRoom - kMany) break;
            }
            if (tid == 0) count = listed;
            __syncthreads();
#pragma unroll 1
            for (int i = 0; i <= E; ++i)
                if (const uint64_t mine = reach(i, key)) {
                    const int at = atomicAdd(&count, 1);
                    if (at < kRoom) list[at] = mine;
                }
            __syncthreads();
            n = min(count, kRoom);
        }
        // (a few chunks' entries are put in order together: 0.5 us of 21 on three chunks)
        if (n > kept && (kept < p.M || n > kMany || chunk == chunks - 1)) {
            for (int i = tid; i < n; i += 256) {
                const uint64_t mine = list[i];
                const int rank = larger_ones(list, n, mine);
                if (rank < p.M) best[rank] = mine;
            }
            __syncthreads();
            kept = min(n, p.M);
            if (tid < kept) list[tid] = best[tid];
            n = kept;
            if (tid == 0) count = kept;
            if (kept == p.M) bound = unordered((uint32_t)(best[p.M - 1] >> 32));
            __syncthreads();
        }
        listed = n;
    }

    const float wave_most = over_wave(most, [](float a, float b) { return max_nan(a, b); });
    const float base = fabsf(wave_most) < INFINITY ? wave_most : 0.f;
    sum = over_wave(sum * exp_behind(most, base), [](float a, float b) { return a + b; });
    if (lane == 0) maxima[wave] = wave_most, sums[wave] = sum;
    __syncthreads();
    // (a row of which a logit is NaN or +infinity has no candidates: its keys are not read)
    uint64_t *out = p.keys + (int64_t)blockIdx.x * p.M;
    if (tid < p.M) out[tid] = tid < kept ? list[tid] : 0;
    if (tid == 64) {
        float m = maxima[0], s = 0.f;
        for (int i = 1; i < 4; ++i) m = max_nan(m, maxima[i]);
        for (int i = 0; i < 4; ++i) s += sums[i] * exp_behind(maxima[i], m);
        p.part_max[blockIdx.x] = m, p.part_sum[blockIdx.x] = s;
    }
}

// One request a workgroup: every beam's sum from its parts, in 64 bits, so that candidates of
// different beams that are close to each other come out in order; then the M best of the parts'
// lists.  All of these are in order: of more than 1024 entries, only the M lists of the best first
// ones count.  A bound as in beam_parts leaves few entries, each of which finds its place by
// counting the larger ones.  What bounds it: the way to memory and back, once where the lists are short
// (5.1 us for one request of 4 beams, 6.7 for 64 of 8; one of 16 beams over 25 parts, 32 taken, 23 by events).
struct BeamEntry {
    double value;    // the candidate, or -infinity
    uint64_t place;  // beam, logit and token (place_of); of equal values the largest comes first; 0: none
    __device__ inline bool operator>(const BeamEntry &o) const { return value > o.value || (value == o.value && place > o.place); }
};
// The lowest beam first, of a beam the largest logit (as in a key), of equal logits the lowest token.  Different
// logits of a beam can be the same value in 64 bits, beside a large score or where they are small beside the log of
// their sum.  The parts' lists are in the order of the logits, and so are the entries; which of a row's parts
// an entry came from makes no difference then.
constexpr int kTokenBits = 19;
static_assert(MONARCH_ATTN_BEAM_MAX_VOCAB <= 1 << kTokenBits && kBeamMax < 1 << (64 - 32 - kTokenBits), "all three in 64 bits");
__device__ inline uint64_t place_of(int beam, uint32_t logit, int token)
{
    return (uint64_t)(kBeamMax - beam) << (32 + kTokenBits) | (uint64_t)logit << kTokenBits | ((1u << kTokenBits) - 1 - (uint32_t)token);
}
__device__ inline int beam_of(uint64_t place) { return kBeamMax - (int)(place >> (32 + kTokenBits)); }
__device__ inline int token_of(uint64_t place) { return (1 << kTokenBits) - 1 - (int)(place & ((1u << kTokenBits) - 1)); }
struct BeamHead {
    BeamEntry e;
    int list;
    __device__ inline bool operator>(const BeamHead &o) const { return e > o.e; }
};
// The upper half of ordered(value), by which entries are bounded; 0: none.
__device__ inline uint32_t height(const BeamEntry &e) { return e.place == 0 ? 0 : (uint32_t)(ordered(e.value) >> 32); }

// A height that M of the workgroup's values at least reach, from the waves' own ones (1 where no wave has M).
__device__ inline uint32_t bound_of(uint32_t x, int m, uint32_t *shared)
{
    const uint32_t mine = reached_by<0>(x, m);
    if (threadIdx.x % 64 == 0) shared[threadIdx.x / 64] = mine;
    __syncthreads();
    return max(max(max(shared[0], shared[1]), max(shared[2], shared[3])), 1u);
}

static __global__ __launch_bounds__(256) void beam_join(BeamSelect p)
{
    constexpr int kAhead = 1024;  // keys that are on their way before the sums are known
    constexpr int kEach = kAhead / 256;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    BeamHead *heads = reinterpret_cast<BeamHead *>(lds);  // of the lists, where there are many
    __shared__ BeamEntry list[kAhead + 8];
    // the log of a beam's sum relative to its largest logit (beside which, of 1e20, 64 bits would not hold it), that logit, its score
    __shared__ double lse[kBeamMax], largest[kBeamMax], score_of[kBeamMax];
    __shared__ int kind[kBeamMax];  // of a beam: 0 candidates by its logits, 1 done, 2 all of them -infinity
    __shared__ int open[kBeamMax];  // the lists that count
    __shared__ uint32_t bounds[2][4];
    __shared__ int count, tops;
    static_assert(kBeamMax * kBeamMax <= kAhead, "entries of the lists that count");
    const int tid = threadIdx.x;
    const int64_t row0 = (int64_t)blockIdx.x * p.K;
    const int lists = p.K * p.parts, all = lists * p.M;
    const uint64_t *keys = p.keys + row0 * p.parts * p.M;
    const bool whole = all <= kAhead;  // else the lists' first entries come first
    uint64_t key[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) key[j] = keys[whole ? min(tid + 256 * j, all - 1) : min(tid + 256 * j, lists - 1) * p.M];
    if (tid == 0) count = 0, tops = 0;
    const int width = p.K <= 4 ? 64 : p.K <= 8 ? 32 : p.K <= 16 ? 16 : 8;  // threads a beam
    if (const int k = tid / width, i0 = tid % width; k < p.K) {
        const int64_t row = row0 + k;
        const float *maxima = p.part_max + row * p.parts, *sums = p.part_sum + row * p.parts;
        // (a beam that is done or not in use has written nothing there: what is read is not taken)
        const float m0 = i0 < p.parts ? maxima[i0] : -INFINITY, s0 = i0 < p.parts ? sums[i0] : 0.f, score = p.scores[row];
        const bool dead = !(score > -INFINITY), ended = p.done && p.done[row];
        float most = m0;
        for (int i = i0 + width; i < p.parts; i += width) most = max_nan(most, maxima[i]);
        for (int s = 1; s < width; s <<= 1) most = max_nan(most, __shfl_xor(most, s));
        const bool fine = fabsf(most) < INFINITY;
        auto weight = [&](float m) { return exp2(((double)m - (double)most) * (double)kLog2e); };
        double sum = s0 * weight(m0);
        for (int i = i0 + width; i < p.parts; i += width) sum += (double)sums[i] * weight(maxima[i]);
        for (int s = 1; s < width; s <<= 1) sum += __shfl_xor(sum, s);
        if (i0 == 0) {
            kind[k] = dead ? 2 : ended ? 1 : fine ? 0 : 2;
            // (in the unit that the exponentials had, kLog2e in 32 bits: off by 2e-8 of the row's entropy)
            lse[k] = log2(sum) / (double)kLog2e;
            largest[k] = most, score_of[k] = score;
        }
    }
    __syncthreads();
    // entry i of list l, of that key, or none
    auto entry = [&](int l, int i, uint64_t key) {
        const int k = l / p.parts;
        BeamEntry e{-(double)INFINITY, 0};
        if (kind[k] == 0) {
            if (key == 0) return e;
            const double x = score_of[k] + (((double)unordered((uint32_t)(key >> 32)) - largest[k]) - lse[k]);
            if (x == x) e.value = x;
            e.place = place_of(k, (uint32_t)(key >> 32), (int)(0xffffffffu - (uint32_t)key));
        } else if (l == k * p.parts && i < p.V) {
            const bool first = kind[k] == 1 && i == 0;  // done: the end token, then the others, in front of it and behind it
            const int t = kind[k] == 2 ? i : first ? p.eos : i - 1 < p.eos ? i - 1 : i;
            if (first) e.value = score_of[k];
            e.place = place_of(k, 0, t);
        }
        return e;
    };
    BeamEntry mine[kEach];
    uint32_t top = 0;
    auto take = [&](int some, auto &&list_of, auto &&number_of) {  // the entries of this thread's keys
        top = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const int x = tid + 256 * j;
            mine[j] = BeamEntry{-(double)INFINITY, 0};
            if (256 * j < some && x < some) mine[j] = entry(list_of(x), number_of(x), key[j]);
            top = max(top, height(mine[j]));
        }
    };
    if (whole) {
        take(all, [&](int x) { return x / p.M; }, [&](int x) { return x % p.M; });
    } else {
        take(lists, [](int x) { return x; }, [](int) { return 0; });
        const uint32_t low = bound_of(top, p.M, bounds[0]);
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (height(mine[j]) >= low) heads[atomicAdd(&tops, 1)] = BeamHead{mine[j], tid + 256 * j};
        __syncthreads();
        const int n = tops;
        for (int i = tid; i < n; i += 256) {
            const int rank = larger_ones(heads, n, heads[i]);
            if (rank < p.M) open[rank] = heads[i].list;
        }
        __syncthreads();
        const int some = min(n, p.M) * p.M;
#pragma unroll
        for (int j = 0; j < kEach; ++j)
            if (const int x = tid + 256 * j; x < some) key[j] = keys[open[x / p.M] * p.M + x % p.M];
        take(some, [&](int x) { return open[x / p.M]; }, [&](int x) { return x % p.M; });
    }
    const uint32_t low = bound_of(top, p.M, bounds[1]);
#pragma unroll
    for (int j = 0; j < kEach; ++j)
        if (height(mine[j]) >= low) list[atomicAdd(&count, 1)] = mine[j];
    __syncthreads();
    const int n = count;
    for (int i = tid; i < n; i += 256) {
        const BeamEntry e = list[i];
        const int rank = larger_ones(list, n, e);
        if (rank >= p.M) continue;
        const int k = beam_of(e.place), t = token_of(e.place);
        const int64_t to = (int64_t)blockIdx.x * p.M + rank;
        p.scores_out[to] = (float)e.value;
        p.tokens[to] = t, p.parents[to] = k;
        if (p.done_out) p.done_out[to] = (p.done && p.done[row0 + k]) || t == p.eos;
    }
}

// The rows of the started page of every beam, and the table's entries of its full pages, from its
// parent, in place: a thread holds the same 16 bytes (the same entry) of all beams of a request, and
// stores none before all are loaded.  So no other thread has a part in what it reads and writes, and
// no copy of the cache is needed.  Beams that are their own parent cost nothing.  What bounds it: bytes (64
// requests of 8 beams, pages of 64 tokens, 8 heads of 128 in bf16, 107 MB both ways: 25 us, 4.2 TB/s; one
// request of 4 beams 3.6 us, latency).
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
