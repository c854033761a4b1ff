// The gradient of exact attention over packed sequences, and of cross attention to the rows of others.
//
// With P = exp(s Q K^T - lse) and the upstream gradient dO:
//   delta_i = sum_c dO_ic O_ic (= sum_j P_ij dP_ij),  dP = dO V^T,
//   dS = P (dP - delta),  dQ = s dS K,  dK = s dS^T Q,  dV = P^T dO,
// dK and dV summed over the query heads of their key head.
//
// A row that sees one key has the weight 1 whatever the score: its dS is zero,
// which dP - delta would give up to rounding only.
//
// Launches: the row statistics; then, in one, dQ, a workgroup per 128 packed rows (fp32: 64)
// that walks the keys, and dK and dV, a workgroup per 64 keys that walks the
// query rows, or several for pieces of them, whose sums a further launch adds up.
// The scores and dP are formed twice (7 products instead of 5), so that each
// sum has one owner that adds in a fixed order in fp32 registers, without atomics.
//
// On 9550 rows of 7 sequences, 16 heads on 4 of 128, bf16, causal (264 GFLOP in 5 products, 370 in
// 7): statistics 23 us (118 MB, 5 TB/s), dQ, dK and dV 420-440 us, sums of the pieces 22 us. The
// matrix units are busy in 37 to 40 % of the cycles and the vector units in 26 to 28 %: what bounds
// it is the chain from scores to dS, with two waves a SIMD to cover it.
#pragma once

#include "seq_attn.hpp"

namespace ma {

// fp16 holds 2^-24 to 65504, and dS is as small as the upstream gradient times
// a weight: dS is formed times a power of two under which its largest possible
// value, 2 |dO_i| max|v_j| over the keys that row i sees, is just below 2^15, and P times 2^14.
// Both are taken out of the fp32 sums.  dQ, whose sums are those of a row, has a power of two a row;
// dK and dV one for the rows that a workgroup walks.  So what a sequence's gradient is depends
// on no other one's.  bf16 and fp32 have the range themselves.
template <typename T> struct BwdScale {
    static constexpr bool kScaled = std::is_same<T, _Float16>::value;
    static constexpr float kP = kScaled ? 14.f : 0.f;  // log2

    // The largest of the norms of `count` rows and `heads` heads from `at` on that this thread of
    // NTH reads: 4 bytes for the 4 D of a row that the walk reads, eight loads on their way at a time.
    // (9550 rows of 7 sequences, 16 heads on 4 of 128: 470 us for 460 with the largest norms of the
    // whole call, one sequence of 16384: 2.21 ms for 2.16.)
    template <int NTH> __device__ static float own_largest(const float *at, int count, int heads, int64_t stride)
    {
        float a = 0.f;
        const uint32_t all = (uint32_t)count * (uint32_t)heads;  // (below 2^31)
        for (uint32_t i = threadIdx.x; i < all; i += 8 * NTH) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint32_t j = min(i + u * NTH, all - 1), head = heads == 1 ? 0 : j / (uint32_t)count;
                x[u] = at[head * stride + (j - head * (uint32_t)count)];
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) a = fmaxf(a, x[u]);
        }
        return a;
    }
    // The largest a and b of the workgroup.
    template <int NTH> __device__ static void all_largest(float &a, float &b, char *lds)
    {
        for (int x = 1; x < 64; x <<= 1) a = fmaxf(a, __shfl_xor(a, x)), b = fmaxf(b, __shfl_xor(b, x));
        float *sh = reinterpret_cast<float *>(lds);
        if (threadIdx.x % 64 == 0) sh[threadIdx.x / 32] = a, sh[threadIdx.x / 32 + 1] = b;
        __syncthreads();
        for (int i = 0; i < NTH / 64; ++i) a = fmaxf(a, sh[2 * i]), b = fmaxf(b, sh[2 * i + 1]);
        __syncthreads();
        a = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(a)));
        b = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(b)));
    }
    // The power of two for rows of dO and v of at most these norms.
    __device__ static float of(float norm_g, float norm_v)
    {
        const float most = 2.f * sqrtf(norm_g) * sqrtf(norm_v);
        const int e = most > 0.f ? 14 - ilogbf(most) : 0;
        return ldexpf(1.f, max(-60, min(e, 60)));
    }
};

// delta and lse in log2 units of every (row, head), 16 lanes a row; in fp16 also
// the norms of dO and v.  A workgroup takes one head of 16 rows at a time, whose lse, delta
// and lse2 are then 64 bytes together.
template <typename T, Keys KEYS> __global__ __launch_bounds__(256) void seq_stats(SeqBwd p)
{
    const Seqs &keys = KEYS == kCross ? p.keys : p.seqs;
    constexpr int V = 16 / (int)sizeof(T);
    const int Hq = p.Hkv * p.G, lane = threadIdx.x & 15;
    if (p.clear) {
        clear_outside<256>(p.seqs, p.dq, (int64_t)Hq * p.d * sizeof(T), blockIdx.x, gridDim.x);
        clear_outside<256>(keys, p.dk, (int64_t)p.Hkv * p.d * sizeof(T), blockIdx.x, gridDim.x);
        clear_outside<256>(keys, p.dv, (int64_t)p.Hkv * p.d * sizeof(T), blockIdx.x, gridDim.x);
    }
    const int first = p.seqs.start(0), last = p.seqs.start(p.seqs.B);  // (rows of no sequence count for nothing)
#pragma unroll 2
    for (int64_t u = blockIdx.x; u < ((int64_t)last - first + 15) / 16 * Hq; u += gridDim.x) {
        const int head = (int)(u % Hq), row = first + (int)(u / Hq) * 16 + (int)(threadIdx.x >> 4);
        if (row >= last) continue;
        const int64_t i = (int64_t)row * Hq + head;
        float sum = 0.f, norm = 0.f;
        for (int col = lane * V; col < p.d; col += 16 * V) {
            T a[V], b[V];
            __builtin_memcpy(a, (const T *)p.out + i * p.d + col, 16);
            __builtin_memcpy(b, (const T *)p.dout + i * p.d + col, 16);
            if (p.rest) {
                T r[V];
                __builtin_memcpy(r, (const T *)p.rest + i * p.d + col, 16);
#pragma unroll
                for (int e = 0; e < V; ++e) sum = __builtin_fmaf((float)r[e], (float)b[e], sum);
            }
#pragma unroll
            for (int e = 0; e < V; ++e) {
                sum = __builtin_fmaf((float)a[e], (float)b[e], sum);
                if constexpr (BwdScale<T>::kScaled) norm = __builtin_fmaf((float)b[e], (float)b[e], norm);
            }
        }
#pragma unroll
        for (int x = 1; x < 16; x <<= 1) {
            sum += __shfl_xor(sum, x);
            if constexpr (BwdScale<T>::kScaled) norm += __shfl_xor(norm, x);
        }
        if (lane == 0) {
            const int64_t at = (int64_t)head * p.seqs.total + row;
            p.delta[at] = sum;
            p.lse2[at] = p.lse[at] * kLog2e;
            if constexpr (BwdScale<T>::kScaled) p.norm_g[at] = norm < INFINITY ? norm : 0.f;
        }
    }
    if constexpr (BwdScale<T>::kScaled) {
        const int first_k = keys.start(0), last_k = keys.start(keys.B);
        for (int64_t u = blockIdx.x; u < ((int64_t)last_k - first_k + 15) / 16 * p.Hkv; u += gridDim.x) {
            const int head = (int)(u % p.Hkv), row = first_k + (int)(u / p.Hkv) * 16 + (int)(threadIdx.x >> 4);
            if (row >= last_k) continue;
            float norm = 0.f;
            const T *v = (const T *)p.v + row * p.ldv + head * p.d;
            for (int col = lane * V; col < p.d; col += 16 * V) {
                T a[V];
                __builtin_memcpy(a, v + col, 16);
#pragma unroll
                for (int e = 0; e < V; ++e) norm = __builtin_fmaf((float)a[e], (float)a[e], norm);
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) norm += __shfl_xor(norm, x);
            if (lane == 0) p.norm_v[(int64_t)head * keys.total + row] = norm < INFINITY ? norm : 0.f;
        }
    }
}

// dQ: the forward's schedule.  S^T = K Q^T and dP^T = V dO^T hold one query row a
// lane, so lse and delta are lane scalars, and dS^T feeds dQ^T += K^T dS^T from registers.
template <typename T, int D, Keys KEYS> struct SeqBwdQ {
    using S = SeqTile<T, D>;
    using frag = typename S::frag;
    static constexpr int W = 4, NTH = 64 * W;
    static constexpr int WR = S::kF32 ? 2 : W, KW = W / WR, R = 32 * WR;  // row blocks by parts of a tile's keys
    static constexpr int BN = 64, KT = BN / 32 / KW;
    static constexpr int TILE = BN * S::ROW;
    static constexpr int LDS_BYTES = 4 * TILE;
    using Copy = TileCopy<T, D, BN, W>;

    template <bool MASK>
    __device__ static void step(const char *kt, const char *vt, const frag *qf, const frag *gf, int see, float c, float lse2,
                                float delta, float scale, f32x16 *dq, int lane)
    {
        // fragments of a 32-key part: the rows of K, the rows of V, the columns of K
        constexpr int NA = S::kF32 ? 0 : 2 * S::ND, NP = 2 * S::NS + NA, N = KT * NP, AHEAD = S::kF32 ? 2 : 4;
        FragStream<frag, N, AHEAD> stream;
        auto load = [&](int u) {
            const int off = u / NP * 32 * S::ROW, i = u % NP;
            if constexpr (!S::kF32)
                if (i >= 2 * S::NS) return S::columns(kt + off + (i - 2 * S::NS) / S::ND * 16 * S::ROW, (i - 2 * S::NS) % S::ND, lane);
            return S::row_frag((i < S::NS ? kt : vt) + off, i % S::NS, lane);
        };
        auto reads = [&](int u) { return u + AHEAD >= N ? 0 : (u + AHEAD) % NP >= 2 * S::NS ? 2 : 1; };
        stream.start(load);
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, AHEAD, 0);
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int i = 0; i < 2 * S::NS; ++i) {
                stream.next(t * NP + i, load, [&](const frag &x) {
                    if (i < S::NS) s = S::M::mma(x, qf[i], s);
                    else dp = S::M::mma(x, gf[i - S::NS], dp);
                });
                sched_step<(S::kF32 ? 4 : 1)>(reads(t * NP + i));
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
                float x = w * (dp[r] - delta);
                if constexpr (BwdScale<T>::kScaled) x *= scale;
                s[r] = MASK && 32 * t + kRow32(r) >= see ? 0.f : x;
            }
            Probs32<T> pf;
            pf.pack(s);
            if constexpr (S::kF32) {
#pragma unroll
                for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        dq[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(S::element(kt, 32 * t + kRow32(r) + 4 * (lane >> 5), dt, lane), pf.s[r], dq[dt], 0, 0, 0);
            } else {
#pragma unroll
                for (int i = 2 * S::NS; i < NP; ++i) {
                    const int ks = (i - 2 * S::NS) / S::ND, dt = (i - 2 * S::NS) % S::ND;
                    stream.next(t * NP + i, load, [&](const frag &x) { dq[dt] = S::M::mma(x, pf.f[ks], dq[dt]); });
                    sched_step<1>(reads(t * NP + i));
                }
            }
        }
    }

    __device__ static void run(const SeqBwd &p, char *lds, int block)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        const int kvh = uniform(block % p.Hkv);
        const int pieces = KEYS == kCross ? p.pieces_q : 1, piece = uniform(block / p.Hkv % pieces);
        const int64_t t = p.tiles_q - 1 - block / p.Hkv / pieces;  // later rows see more keys: they start first
        const int seq = uniform(seq_of_tile(p.seqs, t, p.G, R, lane));
        if (seq < 0) return;
        const int tile = uniform((int)(t - tile0(p.seqs, seq, p.G, R)));
        const int row0 = uniform(p.seqs.start(seq)), n = uniform(p.seqs.length(seq));
        const int key_row0 = KEYS == kCross ? uniform(p.keys.start(seq)) : row0, keys = KEYS == kCross ? uniform(p.keys.count(seq)) : n;
        const int rows = n * p.G, r0 = tile * R, tok0 = r0 / p.G;
        auto visible = [&](int r) { return p.causal ? min(r, rows - 1) / p.G + 1 : keys; };
        // the keys of this piece, whole tiles of them but for the last one's
        const int steps = (uniform(visible(r0 + R - 1)) + BN - 1) / BN;
        const int begin = KEYS == kCross ? uniform((int)((int64_t)steps * piece / pieces)) * BN : 0;
        const int see_all = uniform(visible(r0));
        const int last = KEYS == kCross ? min(see_all, uniform((int)((int64_t)steps * (piece + 1) / pieces)) * BN) : uniform(visible(r0 + R - 1));
        const int wr0 = r0 + wave % WR * 32, part = wave / WR * 32 * KT;
        const int see_most = uniform(visible(wr0 + 31));

        const int r = min(wr0 + (lane & 31), rows - 1);
        const int vis = visible(r), tok = r / p.G - tok0, head = kvh * p.G + r % p.G, Hq = p.Hkv * p.G;
        const Span qs((const T *)p.q + (row0 + tok0) * p.ldq), gs((const T *)p.dout + (int64_t)(row0 + tok0) * Hq * p.d);
        frag qf[S::NS], gf[S::NS];
#pragma unroll
        for (int i = 0; i < S::NS; ++i) {
            const int col = (2 * i + (lane >> 5)) * S::V;
            u32x4 x = qs.load16((tok * (int)p.ldq + head * p.d + col) * (int)sizeof(T), col < p.d);
            __builtin_memcpy(&qf[i], &x, 16);
            x = gs.load16(((tok * Hq + head) * p.d + col) * (int)sizeof(T), col < p.d);
            __builtin_memcpy(&gf[i], &x, 16);
        }
        const int64_t at = (int64_t)head * p.seqs.total + row0 + tok0 + tok;
        const float lse2 = p.lse2[at], delta = p.delta[at];
        float scale = 1.f;  // of this row's dS
        if constexpr (BwdScale<T>::kScaled) {
            float most = BwdScale<T>::template own_largest<NTH>(p.norm_v + (int64_t)kvh * (KEYS == kCross ? p.keys : p.seqs).total + key_row0, KEYS == kCross ? keys : last, 1, 0), none = 0.f;
            BwdScale<T>::template all_largest<NTH>(most, none, lds);
            scale = BwdScale<T>::of(p.norm_g[at], most);
        }

        const int ldk = (int)p.ldk * (int)sizeof(T), ldv = (int)p.ldv * (int)sizeof(T);
        const T *k = (const T *)p.k + key_row0 * p.ldk + kvh * p.d, *v = (const T *)p.v + key_row0 * p.ldv + kvh * p.d;
        Copy ck, cv;
        ck.init(ldk, p.d, wave, lane);
        cv.init(ldv, p.d, wave, lane);
        auto bring = [&](int key0, int buf) {
            if (key0 >= last) return;
            ck.tile(k + key0 * p.ldk, keys - key0, ldk, lds + 2 * TILE * buf, wave);
            cv.tile(v + key0 * p.ldv, keys - key0, ldv, lds + 2 * TILE * buf + TILE, wave);
        };

        f32x16 dq[S::ND];
#pragma unroll
        for (int dt = 0; dt < S::ND; ++dt) dq[dt] = f32x16{};
        bring(begin, 0);
        int key0 = begin, buf = 0;
        // (a copy of the step for each buffer: its LDS addresses are constants)
        const int whole = min(see_all, last) - BN;
        auto unmasked = [&](int b) {
            tile_barrier();
            bring(key0 + BN, b ^ 1);
            step<false>(lds + 2 * TILE * b + part * S::ROW, lds + 2 * TILE * b + TILE + part * S::ROW, qf, gf, 0, p.c, lse2, delta, scale, dq, lane);
            key0 += BN, buf = b ^ 1;
        };
#pragma unroll 1
        while (key0 <= whole) {
            unmasked(0);
            if (key0 <= whole) unmasked(1);
        }
#pragma unroll 1
        for (; key0 < last; key0 += BN, buf ^= 1) {
            tile_barrier();
            bring(key0 + BN, buf ^ 1);
            if (key0 + part < see_most)
                step<true>(lds + 2 * TILE * buf + part * S::ROW, lds + 2 * TILE * buf + TILE + part * S::ROW, qf, gf,
                           vis - key0 - part - 4 * (lane >> 5), p.c, lse2, delta, scale, dq, lane);
        }
        if constexpr (KW > 1) {  // the waves' sums over their keys, into the first ones'
            static_assert((KW - 1) * WR * S::ND * 16 * 256 <= LDS_BYTES, "the tiles' room holds them");
            float *sh = reinterpret_cast<float *>(lds) + lane;
            __syncthreads();
            if (wave >= WR)
#pragma unroll
                for (int i = 0; i < S::ND * 16; ++i) sh[((wave - WR) * S::ND * 16 + i) * 64] = dq[i / 16][i % 16];
            __syncthreads();
            if (wave >= WR) return;
#pragma unroll
            for (int w = 1; w < KW; ++w)
#pragma unroll
                for (int i = 0; i < S::ND * 16; ++i) dq[i / 16][i % 16] += sh[(((w - 1) * WR + wave) * S::ND * 16 + i) * 64];
        }
        const float by = vis == 1 ? 0.f : p.c * kLn2 / scale;
        if constexpr (KEYS == kCross)
            if (pieces > 1) {
                const Span ps(p.part_q + ((int64_t)piece * p.seqs.total + row0 + tok0) * Hq * D);
                store_row<float, S::ND>(ps, dq, by, (tok * Hq + head) * D, D, wr0 + (lane & 31) < rows, lane);
                return;
            }
        const Span os((T *)p.dq + (int64_t)(row0 + tok0) * Hq * p.d);
        store_row<T, S::ND>(os, dq, by, (tok * Hq + head) * p.d, p.d, wr0 + (lane & 31) < rows, lane);
    }
};

// dK and dV: one workgroup per R = 64 keys of a key head, which walks the query
// rows of the group's heads in tiles of 32 NQ.  Wave (kb, qb) takes key block kb
// and the tile's rows 32 qb on; the NQ sums of a key block are added up at the end.
// S = Q K^T and dP = dO V^T hold one key a lane, so P and dS feed
// dV^T += dO^T P and dK^T += Q^T dS from registers.
//
// A key block is 32 keys, so that K, dK and dV of it leave room for a second
// wave on the SIMD (past D = 64 with V read from LDS); of 64 keys they take all registers, and
// what does not fit goes through memory (530 us on the rows above; 288 us so, as a launch of
// its own).  Few keys and many rows a workgroup, because the
// longest walk, that of a long sequence's first keys, bounds the call.
template <typename T, int D, Keys KEYS> struct SeqBwdK {
    using S = SeqTile<T, D>;
    using frag = typename S::frag;
    static constexpr int NK = 2, NQ = 2, W = NK * NQ, NTH = 64 * W, R = 32 * NK;
    static constexpr int BQ = 32 * NQ, TILE = BQ * S::ROW;
    static constexpr bool kVInLds = !S::kF32 && D > 64;
    static constexpr int LDS_BYTES = 4 * TILE + (kVInLds ? R * S::ROW : 0);
    using Copy = TileCopy<T, D, BQ, W>;

    struct Grads {
        f32x16 dk[S::ND], dv[S::ND];
    };

    // 32 rows of Q and dO (qt, gt); terms: -lse / s, so that P = exp2(c S), and -delta of the
    // rows.  `ahead`: the first of them minus this lane's key; rows before `first` (row 0, which
    // sees one key) pass no gradient to scores. vt: the key block's V rows in LDS, where they are
    // there.
    template <bool MASK>
    __device__ static void step(const char *qt, const char *gt, const RowTerms<T> &terms, const frag *kf, const frag *vf,
                                const char *vt, int ahead, int first, float c, float scale, Grads &x, int lane)
    {
        // fragments: the rows of Q, then of dO (each with V's behind it), then the columns of dO
        // and of Q
        constexpr int NV = kVInLds ? 2 : 1, NR = (1 + NV) * S::NS, NA = S::kF32 ? 0 : 2 * S::ND, N = NR + 2 * NA, AHEAD = S::kF32 || D > 96 ? 2 : 4;
        FragStream<frag, N, AHEAD> stream;
        auto load = [&](int u) {
            if constexpr (!S::kF32)
                if (u >= NR) {
                    const int i = (u - NR) % NA;
                    return S::columns((u < NR + NA ? gt : qt) + i / S::ND * 16 * S::ROW, i % S::ND, lane);
                }
            const int i = (u - S::NS) / NV;
            return u < S::NS ? S::row_frag(qt, u, lane) : S::row_frag((u - S::NS) % NV ? vt : gt, i, lane);
        };
        auto reads = [&](int u) { return u + AHEAD >= N ? 0 : u + AHEAD >= NR ? 2 : 1; };
        stream.start(load);
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, AHEAD, 0);
        // In fp32 a sum that starts at lse rounds at lse's size all the way (16 rows over 700 keys of 128 columns: dK and
        // dV are off by 2.0e-6, with lse added last by 0.7e-6). Packed calls keep the order, and so the bits, that they have.
        constexpr bool kLast = S::kF32 && KEYS == kCross;
        f32x16 s = kLast ? f32x16{} : terms.template add<0>(f32x16{}, lane), dp = terms.template add<1>(f32x16{}, lane);
#pragma unroll
        for (int u = 0; u < S::NS; ++u) {
            stream.next(u, load, [&](const frag &y) { s = S::M::mma(y, kf[u], s); });
            sched_step<(S::kF32 ? 4 : 1)>(reads(u));
        }
        if constexpr (kLast) s = terms.template add<0>(s, lane);
#pragma unroll
        for (int i = 0; i < S::NS; ++i) {
            const int u = S::NS + i * NV;
            frag g;
            stream.next(u, load, [&](const frag &y) { g = y; });
            if constexpr (kVInLds) {
                stream.next(u + 1, load, [&](const frag &y) { dp = S::M::mma(g, y, dp); });
                sched_step<1>(u + 1 + AHEAD >= NR ? 2 : 1);
            } else {
                dp = S::M::mma(g, vf[i], dp);
                sched_step<(S::kF32 ? 4 : 1)>(reads(u));
            }
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = kRow32(r) + 4 * (lane >> 5);
            float w = __builtin_amdgcn_exp2f(s[r] * c);
            if (MASK && row + ahead < 0) w = 0.f;
            float y = w * dp[r];
            if constexpr (BwdScale<T>::kScaled) y *= scale;
            s[r] = w;
            dp[r] = MASK && (row + ahead < 0 || row < first) ? 0.f : y;
        }
        Probs32<T> pf, sf;
        pf.pack(s);
        sf.pack(dp);
        if constexpr (S::kF32) {
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int row = kRow32(r) + 4 * (lane >> 5);
                    x.dv[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(S::element(gt, row, dt, lane), pf.s[r], x.dv[dt], 0, 0, 0);
                    x.dk[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(S::element(qt, row, dt, lane), sf.s[r], x.dk[dt], 0, 0, 0);
                }
        } else {
#pragma unroll
            for (int u = NR; u < N; ++u) {
                const int i = (u - NR) % NA, ks = i / S::ND, dt = i % S::ND;
                stream.next(u, load, [&](const frag &y) {
                    if (u < NR + NA) x.dv[dt] = S::M::mma(y, pf.f[ks], x.dv[dt]);
                    else x.dk[dt] = S::M::mma(y, sf.f[ks], x.dk[dt]);
                });
                sched_step<1>(reads(u));
            }
        }
    }

    // The waves' sums of one gradient, scaled, to the keys' rows of `out`; zero in the `padding` rows behind them.
    template <typename O>
    __device__ static void add_up(char *lds, const f32x16 *x, const Span &out, float by, int ld, int d, int keys, int padding, int wave, int lane)
    {
        constexpr int N = S::ND * 4 * 64;  // a wave's sums, in 4 values
        static_assert(W * N * 16 <= 4 * TILE, "the tiles' room holds them");
        f32x4 *mine = reinterpret_cast<f32x4 *>(lds) + wave * N + lane;
        __syncthreads();
#pragma unroll
        for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine[(dt * 4 + e) * 64] = f32x4{x[dt][4 * e], x[dt][4 * e + 1], x[dt][4 * e + 2], x[dt][4 * e + 3]};
        __syncthreads();
        for (int i = wave; i < NK * S::ND; i += W) {
            const int kb = i / S::ND, dt = i % S::ND;
            const f32x4 *src = reinterpret_cast<const f32x4 *>(lds) + kb * N + dt * 256 + lane;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f32x4 sum = src[e * 64];
#pragma unroll
                for (int q = 1; q < NQ; ++q) sum += src[q * NK * N + e * 64];
                const int key = 32 * kb + (lane & 31), col = 32 * dt + 8 * e + 4 * (lane >> 5);
                if constexpr (KEYS == kCross)
                    if (key >= keys) sum = f32x4{0.f, 0.f, 0.f, 0.f};
                out.store<O>(sum * by, (key * ld + col) * (int)sizeof(O), key < keys + padding && col < d);
            }
        }
    }

    __device__ static void run(const SeqBwd &p, char *lds, int block)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), kb = wave % NK, qb = wave / NK;
        const int kvh = uniform(block % p.Hkv);
        const int64_t t = block / p.Hkv / p.pieces;  // (earlier keys are seen by more rows: they start first)
        const int piece = uniform(block / p.Hkv % p.pieces);
        const Seqs &key_seqs = KEYS == kCross ? p.keys : p.seqs;
        const int seq = uniform(seq_of_tile(key_seqs, t, 1, R, lane));
        if (seq < 0) return;
        const int row0 = uniform(p.seqs.start(seq)), n = uniform(p.seqs.length(seq));
        // keys: of the sequence; behind them come `padding` rows, whose gradients are zero
        const int key_row0 = KEYS == kCross ? uniform(p.keys.start(seq)) : row0, keys = KEYS == kCross ? uniform(p.keys.count(seq)) : n;
        const int k0 = uniform((int)(t - tile0(key_seqs, seq, 1, R)) * R), Hq = p.Hkv * p.G;
        const int padding = KEYS == kCross ? uniform(p.keys.length(seq)) - max(keys, k0) : 0;
        const int from = p.causal ? k0 : 0;  // the first row that sees a key of this workgroup
        float ds = 1.f;                      // the power of two of dS
        if constexpr (BwdScale<T>::kScaled) {
            const float *g = p.norm_g + (int64_t)kvh * p.G * p.seqs.total + row0 + from, *v = p.norm_v + (int64_t)kvh * key_seqs.total + key_row0;
            float most_g = BwdScale<T>::template own_largest<NTH>(g, n - from, p.G, p.seqs.total);
            float most_v = BwdScale<T>::template own_largest<NTH>(v, keys, 1, 0);
            BwdScale<T>::template all_largest<NTH>(most_g, most_v, lds);
            ds = BwdScale<T>::of(most_g, most_v);
        }

        const Span ks((const T *)p.k + (key_row0 + k0) * p.ldk + kvh * p.d), vs((const T *)p.v + (key_row0 + k0) * p.ldv + kvh * p.d);
        const int ldv = (int)p.ldv * (int)sizeof(T), kc = max(0, min(32 * kb + (lane & 31), keys - 1 - k0));
        char *vt = lds + 4 * TILE;
        frag kf[S::NS], vf[kVInLds ? 1 : S::NS];
        if constexpr (kVInLds) {
            TileCopy<T, D, R, W> cv;
            cv.init(ldv, p.d, wave, lane);
            cv.tile((const T *)p.v + (key_row0 + k0) * p.ldv + kvh * p.d, keys - k0, ldv, vt, wave);
        }
#pragma unroll
        for (int i = 0; i < S::NS; ++i) {
            const int col = (2 * i + (lane >> 5)) * S::V;
            u32x4 x = ks.load16((kc * (int)p.ldk + col) * (int)sizeof(T), col < p.d);
            __builtin_memcpy(&kf[i], &x, 16);
            if constexpr (!kVInLds) {
                x = vs.load16(kc * ldv + col * (int)sizeof(T), col < p.d);
                __builtin_memcpy(&vf[i], &x, 16);
            }
        }

        const int ldq = (int)p.ldq * (int)sizeof(T), ldg = Hq * p.d * (int)sizeof(T);
        Copy cq, cg;
        cq.init(ldq, p.d, wave, lane);
        cg.init(ldg, p.d, wave, lane);
        // The walk: every head's tiles from row `from` on, this piece's share of them.
        const int tiles = KEYS == kCross && keys <= k0 ? 0 : (n - from + BQ - 1) / BQ;
        const int begin = uniform((int)((int64_t)p.G * tiles * piece / p.pieces)), end = uniform((int)((int64_t)p.G * tiles * (piece + 1) / p.pieces));
        float lse2 = 0.f, delta = 0.f;  // of this lane's row of the tile that is copied
        auto bring = [&](int i, int g, int q0, int buf) {  // tile i of the walk, at row q0 of head g or the next one's first
            if (i >= end) return;
            if (q0 >= n) q0 = from, ++g;
            const int head = kvh * p.G + g;
            char *to = lds + 2 * TILE * buf;
            cq.tile((const T *)p.q + (row0 + q0) * p.ldq + head * p.d, n - q0, ldq, to, wave);
            cg.tile((const T *)p.dout + ((int64_t)(row0 + q0) * Hq + head) * p.d, n - q0, ldg, to + TILE, wave);
            const int r = min(q0 + 32 * qb + (lane & 31), n - 1);
            const int64_t at = (int64_t)head * p.seqs.total + row0 + r;
            lse2 = p.lse2[at], delta = p.delta[at];
            if (q0 + 32 * qb + (lane & 31) >= n) lse2 = 1e30f, delta = 0.f;  // a row that is not there has weights of zero
        };
        const float per_c = 1.f / p.c;
        RowTerms<T> terms;

        Grads x;
#pragma unroll
        for (int dt = 0; dt < S::ND; ++dt) x.dk[dt] = x.dv[dt] = f32x16{};
        const float scale = BwdScale<T>::kScaled ? ds * 0x1p-14f : 1.f;
        int buf = 0, i = begin, g = KEYS == kCross && tiles == 0 ? 0 : begin / tiles;
        int q0 = from + (begin - g * tiles) * BQ;
        bring(i, g, q0, 0);
        const char *own = lds + 32 * qb * S::ROW, *vrows = vt + 32 * kb * S::ROW;
#pragma unroll 1
        while (i < end) {
            if (q0 >= n) q0 = from, ++g;
            if (p.causal && q0 == from) {  // a head's first tile holds rows that see a part of the keys
                tile_barrier();
                terms.set((BwdScale<T>::kP - lse2) * per_c, -delta, lane);
                bring(i + 1, g, q0 + BQ, buf ^ 1);
                if (q0 + 32 * qb < n)
                    step<true>(own + 2 * TILE * buf, own + 2 * TILE * buf + TILE, terms, kf, vf, vrows,
                               q0 + 32 * qb - k0 - 32 * kb - (lane & 31), 1 - q0 - 32 * qb, p.c, scale, x, lane);
                ++i, q0 += BQ, buf ^= 1;
            }
#pragma unroll 1
            for (; i < end && q0 < n; ++i, q0 += BQ, buf ^= 1) {
                tile_barrier();
                terms.set((BwdScale<T>::kP - lse2) * per_c, -delta, lane);
                bring(i + 1, g, q0 + BQ, buf ^ 1);
                if (q0 + 32 * qb < n)
                    step<false>(own + 2 * TILE * buf, own + 2 * TILE * buf + TILE, terms, kf, vf, vrows, 0, 0, p.c, scale, x, lane);
            }
        }
        const float by_k = keys == 1 ? 0.f : p.c * kLn2 / ds, by_v = BwdScale<T>::kScaled ? 0x1p-14f : 1.f;
        if (p.pieces > 1) {
            const int64_t at = (((int64_t)piece * key_seqs.total + key_row0 + k0) * p.Hkv + kvh) * D;
            add_up<float>(lds, x.dk, Span(p.part_k + at), by_k, p.Hkv * D, D, max(0, keys - k0), padding, wave, lane);
            add_up<float>(lds, x.dv, Span(p.part_v + at), by_v, p.Hkv * D, D, max(0, keys - k0), padding, wave, lane);
            return;
        }
        const int64_t out0 = ((int64_t)(key_row0 + k0) * p.Hkv + kvh) * p.d;
        add_up<T>(lds, x.dk, Span((T *)p.dk + out0), by_k, p.Hkv * p.d, p.d, max(0, keys - k0), padding, wave, lane);
        add_up<T>(lds, x.dv, Span((T *)p.dv + out0), by_v, p.Hkv * p.d, p.d, max(0, keys - k0), padding, wave, lane);
    }
};

// Both in one launch, dQ first: its longest walks, over all keys of a long sequence, start at once,
// and the shorter ones of dK and dV fill what they leave free.  (fp32, 6 sequences of up to 1000
// tokens, 12 heads of 64: 98 us, two launches 132 (87 since); the rows above 466 us, two launches
// 474, dK and dV first 472.)
template <typename T, int D, Keys KEYS> __global__ __launch_bounds__(256, sizeof(T) == 4 && D > 64 ? 1 : 2) void seq_bwd(SeqBwd p, int blocks_q)
{
    using K = SeqBwdK<T, D, KEYS>;
    using Q = SeqBwdQ<T, D, KEYS>;
    static_assert(K::NTH == 256 && Q::NTH == 256, "one launch");
    __shared__ __attribute__((aligned(16))) char lds[K::LDS_BYTES > Q::LDS_BYTES ? K::LDS_BYTES : Q::LDS_BYTES];
    const int block = blockIdx.x;
    if (block < blocks_q)
        Q::run(p, lds, block);
    else
        K::run(p, lds, block - blocks_q);
}

// The pieces' sums added up, four columns a thread: dK and dV, and of cross attention dQ.
template <typename T, int D, Keys KEYS> __global__ __launch_bounds__(256) void seq_bwd_join(SeqBwd p)
{
    constexpr int C = D / 4;
    if constexpr (KEYS == kCross) {
        const int Hq = p.Hkv * p.G;
        const int64_t first = (int64_t)p.seqs.start(0) * Hq, rows = p.pieces_q == 1 ? 0 : (int64_t)p.seqs.start(p.seqs.B) * Hq - first;
        const int64_t each = (int64_t)p.seqs.total * Hq * D;
        for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * C; i += (int64_t)gridDim.x * 256) {
            const int64_t row = first + i / C;
            const int col = (int)(i % C) * 4;
            if (col >= p.d) continue;
            const float *q = p.part_q + row * D + col;
            f32x4 a = *(const f32x4 *)q;
            for (int x = 1; x < p.pieces_q; ++x) a += *(const f32x4 *)(q + x * each);
            store4<T>((T *)p.dq + row * p.d + col, a);
        }
        if (p.pieces == 1) return;
    }
    const Seqs &keys = KEYS == kCross ? p.keys : p.seqs;
    const int64_t first = (int64_t)keys.start(0) * p.Hkv, rows = (int64_t)keys.start(keys.B) * p.Hkv - first;
    const int64_t each = (int64_t)keys.total * p.Hkv * D;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * C; i += (int64_t)gridDim.x * 256) {
        const int64_t row = first + i / C;
        const int col = (int)(i % C) * 4;
        if (col >= p.d) continue;
        const float *k = p.part_k + row * D + col, *v = p.part_v + row * D + col;
        f32x4 a = *(const f32x4 *)k, b = *(const f32x4 *)v;
        for (int x = 1; x < p.pieces; ++x) a += *(const f32x4 *)(k + x * each), b += *(const f32x4 *)(v + x * each);
        store4<T>((T *)p.dk + row * p.d + col, a);
        store4<T>((T *)p.dv + row * p.d + col, b);
    }
}

}  // namespace ma
