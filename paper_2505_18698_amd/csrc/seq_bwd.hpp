// The gradient of exact attention over packed sequences.
//
// With P = exp(s Q K^T - lse) and the upstream gradient dO:
//   delta_i = sum_c dO_ic O_ic (= sum_j P_ij dP_ij),  dP = dO V^T,
//   dS = P (dP - delta),  dQ = s dS K,  dK = s dS^T Q,  dV = P^T dO,
// dK and dV summed over the query heads of their key head.
//
// A row that sees one key has the weight 1 whatever the score: its dS is zero,
// which dP - delta would give up to rounding only.
//
// Three launches: the row statistics; dK and dV, a workgroup per 64 keys (32 in fp32) that
// walks the query rows; dQ, a workgroup per 128 packed rows that walks the
// keys.  The scores and dP are formed twice (7 products instead of 5), so that
// each sum has one owner that adds in a fixed order in fp32 registers: no
// atomics, no partial sums in memory.
#pragma once

#include "seq_attn.hpp"

namespace ma {

// fp16 holds 2^-24 to 65504, and dS is as small as the upstream gradient times
// a weight: dS is formed times a power of two under which its largest possible
// value, 2 max|dO_i| max|v_j|, is just below 2^15, and P times 2^14.  Both are
// taken out of the fp32 sums.  bf16 and fp32 have the range themselves.
template <typename T> struct BwdScale {
    static constexpr bool kScaled = std::is_same<T, _Float16>::value;
    static constexpr float kP = kScaled ? 14.f : 0.f;  // log2
    float ds = 1.f;                                    // of dS
    __device__ void find(const SeqBwd &p, char *lds)
    {
        if constexpr (kScaled) {
            float a = 0.f, b = 0.f;
            for (int i = threadIdx.x; i < p.norm_blocks; i += 256) {
                const float2 x = p.norms[i];
                a = fmaxf(a, x.x), b = fmaxf(b, x.y);
            }
            for (int x = 1; x < 64; x <<= 1) a = fmaxf(a, __shfl_xor(a, x)), b = fmaxf(b, __shfl_xor(b, x));
            float *sh = reinterpret_cast<float *>(lds);
            if (threadIdx.x % 64 == 0) sh[threadIdx.x / 64] = a, sh[4 + threadIdx.x / 64] = b;
            __syncthreads();
            a = fmaxf(fmaxf(sh[0], sh[1]), fmaxf(sh[2], sh[3]));
            b = fmaxf(fmaxf(sh[4], sh[5]), fmaxf(sh[6], sh[7]));
            __syncthreads();
            const float most = 2.f * sqrtf(a) * sqrtf(b);
            const int e = most > 0.f ? 14 - ilogbf(most) : 0;
            ds = uniform_float(ldexpf(1.f, max(-60, min(e, 60))));
        }
    }
    __device__ static float uniform_float(float x) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(x))); }
};

// delta and lse in log2 units of every (row, head), 16 lanes a row; in fp16 also the largest norms.
template <typename T> __global__ __launch_bounds__(256) void seq_stats(SeqBwd p)
{
    constexpr int V = 16 / (int)sizeof(T);
    const int Hq = p.Hkv * p.G, lane = threadIdx.x & 15;
    const int first = p.seqs.start(0), last = p.seqs.start(p.seqs.B);  // (rows of no sequence count for nothing)
    const int64_t step = (int64_t)gridDim.x * 16, own = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    float most_g = 0.f, most_v = 0.f;
    for (int64_t i = (int64_t)first * Hq + own; i < (int64_t)last * Hq; i += step) {
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
            const int64_t at = i % Hq * p.seqs.total + i / Hq;
            p.delta[at] = sum;
            p.lse2[at] = p.lse[at] * kLog2e;
        }
        if (norm < INFINITY) most_g = fmaxf(most_g, norm);
    }
    if constexpr (BwdScale<T>::kScaled) {
        for (int64_t i = (int64_t)first * p.Hkv + own; i < (int64_t)last * p.Hkv; i += step) {
            float norm = 0.f;
            const T *v = (const T *)p.v + i / p.Hkv * p.ldv + i % p.Hkv * p.d;
            for (int col = lane * V; col < p.d; col += 16 * V) {
                T a[V];
                __builtin_memcpy(a, v + col, 16);
#pragma unroll
                for (int e = 0; e < V; ++e) norm = __builtin_fmaf((float)a[e], (float)a[e], norm);
            }
#pragma unroll
            for (int x = 1; x < 16; x <<= 1) norm += __shfl_xor(norm, x);
            if (norm < INFINITY) most_v = fmaxf(most_v, norm);
        }
        __shared__ float sh[2][4];
        for (int x = 16; x < 64; x <<= 1) most_g = fmaxf(most_g, __shfl_xor(most_g, x)), most_v = fmaxf(most_v, __shfl_xor(most_v, x));
        if (threadIdx.x % 64 == 0) sh[0][threadIdx.x / 64] = most_g, sh[1][threadIdx.x / 64] = most_v;
        __syncthreads();
        if (threadIdx.x == 0)
            p.norms[blockIdx.x] = float2{fmaxf(fmaxf(sh[0][0], sh[0][1]), fmaxf(sh[0][2], sh[0][3])),
                                         fmaxf(fmaxf(sh[1][0], sh[1][1]), fmaxf(sh[1][2], sh[1][3]))};
    }
}

// One row (lane % 32) of X^T, held as 32 x 32 results, to row `at` elements behind `base` of a [*, d] tensor.
template <typename T, int ND>
__device__ inline void store_transposed(const Span &s, const f32x16 *x, float by, int at, int d, bool real, int lane)
{
#pragma unroll
    for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int col = 32 * dt + 8 * e + 4 * (lane >> 5);
            s.store<T>(f32x4{x[dt][4 * e] * by, x[dt][4 * e + 1] * by, x[dt][4 * e + 2] * by, x[dt][4 * e + 3] * by},
                       (at + col) * (int)sizeof(T), real && col < d);
        }
}

// dQ: the forward's schedule.  S^T = K Q^T and dP^T = V dO^T hold one query row a
// lane, so lse and delta are lane scalars, and dS^T feeds dQ^T += K^T dS^T from registers.
template <typename T, int D> struct SeqBwdQ {
    using S = SeqTile<T, D>;
    using frag = typename S::frag;
    static constexpr int W = 4, NTH = 64 * W, R = 32 * W;
    static constexpr int BN = S::kF32 ? 32 : 64, KT = BN / 32;
    static constexpr int TILE = BN * S::ROW;
    static constexpr int LDS_BYTES = 4 * TILE;
    using Copy = TileCopy<T, D, BN, W>;

    template <bool MASK>
    __device__ static void step(const char *kt, const char *vt, const frag *qf, const frag *gf, int see, float c, float lse2,
                                float delta, float scale, f32x16 (*dq)[S::ND], int lane)
    {
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            f32x16 s = S::scores(kt + t * 32 * S::ROW, qf, lane, f32x16{});
            const f32x16 dp = S::scores(vt + t * 32 * S::ROW, gf, lane, f32x16{});
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2));
                float x = w * (dp[r] - delta);
                if constexpr (BwdScale<T>::kScaled) x *= scale;
                s[r] = MASK && 32 * t + kRow32(r) >= see ? 0.f : x;
            }
            Probs32<T> pf;
            pf.pack(s);
            aggregate<T, D, 1>(kt + t * 32 * S::ROW, &pf, dq, lane);
        }
    }

    __device__ static void run(const SeqBwd &p, char *lds)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        BwdScale<T> sc;
        sc.find(p, lds);
        const int kvh = uniform((int)(blockIdx.x % p.Hkv));
        const int64_t t = p.tiles_q - 1 - (int)(blockIdx.x / p.Hkv);  // later rows see more keys: they start first
        const int seq = uniform(seq_of_tile(p.seqs, t, p.G, R, lane));
        if (seq < 0) return;
        const int tile = uniform((int)(t - tile0(p.seqs, seq, p.G, R)));
        const int row0 = uniform(p.seqs.start(seq)), n = uniform(p.seqs.length(seq));
        const int rows = n * p.G, r0 = tile * R, tok0 = r0 / p.G;
        auto visible = [&](int r) { return p.causal ? min(r, rows - 1) / p.G + 1 : n; };
        const int see_all = uniform(visible(r0)), last = uniform(visible(r0 + R - 1));
        const int see_most = uniform(visible(r0 + wave * 32 + 31));

        const int r = min(r0 + wave * 32 + (lane & 31), rows - 1);
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

        const int ldk = (int)p.ldk * (int)sizeof(T), ldv = (int)p.ldv * (int)sizeof(T);
        const T *k = (const T *)p.k + row0 * p.ldk + kvh * p.d, *v = (const T *)p.v + row0 * p.ldv + kvh * p.d;
        Copy ck, cv;
        ck.init(ldk, p.d, wave, lane);
        cv.init(ldv, p.d, wave, lane);
        auto bring = [&](int key0, int buf) {
            if (key0 >= last) return;
            ck.tile(k + key0 * p.ldk, n - key0, ldk, lds + 2 * TILE * buf, wave);
            cv.tile(v + key0 * p.ldv, n - key0, ldv, lds + 2 * TILE * buf + TILE, wave);
        };

        f32x16 dq[1][S::ND];
#pragma unroll
        for (int dt = 0; dt < S::ND; ++dt) dq[0][dt] = f32x16{};
        bring(0, 0);
        int key0 = 0, buf = 0;
#pragma unroll 1
        for (; key0 + BN <= min(see_all, last); key0 += BN, buf ^= 1) {
            tile_barrier();
            bring(key0 + BN, buf ^ 1);
            step<false>(lds + 2 * TILE * buf, lds + 2 * TILE * buf + TILE, qf, gf, 0, p.c, lse2, delta, sc.ds, dq, lane);
        }
#pragma unroll 1
        for (; key0 < last; key0 += BN, buf ^= 1) {
            tile_barrier();
            bring(key0 + BN, buf ^ 1);
            if (key0 < see_most)
                step<true>(lds + 2 * TILE * buf, lds + 2 * TILE * buf + TILE, qf, gf, vis - key0 - 4 * (lane >> 5), p.c, lse2,
                           delta, sc.ds, dq, lane);
        }
        const Span os((T *)p.dq + (int64_t)(row0 + tok0) * Hq * p.d);
        store_transposed<T, S::ND>(os, dq[0], vis == 1 ? 0.f : p.c * kLn2 / sc.ds, (tok * Hq + head) * p.d, p.d, r0 + wave * 32 + (lane & 31) < rows, lane);
    }
};

// dK and dV: one workgroup per R = 32 KB keys of a key head, whose K and V rows
// every wave keeps in registers as right operands.  The waves divide the query
// rows of the group's heads among them in tiles of 32, each with its own copies
// and without a barrier, and add up their sums at the end.  S = Q K^T and dP = dO V^T hold one key a
// lane, so P and dS feed dV^T += dO^T P and dK^T += Q^T dS from registers.
//
// A tile is read from LDS twice as rows and twice as columns, 32 D bytes each
// in 16-bit types, for 4 KB 32 x 32 x D products: with one key block a wave
// (KB = 1) the LDS is busy longer than the matrix pipes, with two it is not.  The price
// is the registers of a wave per SIMD (K, V, dK and dV of 64 keys: 384 at D = 128).
template <typename T, int D> struct SeqBwdK {
    using S = SeqTile<T, D>;
    using frag = typename S::frag;
    static constexpr int W = S::kF32 && D > 64 ? 2 : 4, NTH = 64 * W, KB = S::kF32 ? 1 : 2, R = 32 * KB;
    static constexpr int TILE = 32 * S::ROW, STATS = 64 * 4;
    static constexpr int OWN = 4 * TILE + STATS;  // a wave's: Q and dO, two of each, and a tile's lse and delta
    static constexpr int LDS_BYTES = W * OWN;
    using Copy = TileCopy<T, D, 32, 1>;

    struct Grads {
        f32x16 dk[KB][S::ND], dv[KB][S::ND];
    };

    // `ahead`: first query row of the tile minus this lane's key of the first
    // block; rows of the tile before `first` (row 0, which sees one key) pass no gradient to scores
    template <bool MASK>
    __device__ static void step(const char *qt, const char *gt, const float *stats, const frag (*kf)[S::NS], const frag (*vf)[S::NS],
                                int ahead, int first, float c, float scale, Grads &x, int lane)
    {
        Probs32<T> pf[KB], sf[KB];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            f32x16 s = S::scores(qt, kf[b], lane, f32x16{});
            f32x16 dp = S::scores(gt, vf[b], lane, f32x16{});
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x4 lse2 = *reinterpret_cast<const f32x4 *>(stats + 8 * e + 4 * (lane >> 5));
                const f32x4 delta = *reinterpret_cast<const f32x4 *>(stats + 32 + 8 * e + 4 * (lane >> 5));
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 4 * e + i, at = kRow32(r) + 4 * (lane >> 5) + ahead - 32 * b;  // query row minus key
                    float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -lse2[i]));
                    if (MASK && at < 0) w = 0.f;
                    float y = w * (dp[r] - delta[i]);
                    if constexpr (BwdScale<T>::kScaled) y *= scale;
                    s[r] = w;
                    dp[r] = MASK && (at < 0 || kRow32(r) + 4 * (lane >> 5) < first) ? 0.f : y;
                }
            }
            pf[b].pack(s);
            sf[b].pack(dp);
            if constexpr (KB > 1) __builtin_amdgcn_sched_barrier(0);  // one block's scores at a time: the registers hold no more
        }
        aggregate<T, D, KB>(gt, pf, x.dv, lane);
        aggregate<T, D, KB>(qt, sf, x.dk, lane);
    }

    // The waves' sums of one gradient, scaled, to the keys' rows of `out`.
    __device__ static void add_up(char *lds, const f32x16 (*x)[S::ND], const Span &out, float by, int at, int d, int keys, int wave, int lane)
    {
        constexpr int N = KB * S::ND * 16 * 64;  // a wave's values
        static_assert(W * N * 4 <= LDS_BYTES, "the tiles' room holds them");
        f32x4 *mine = reinterpret_cast<f32x4 *>(lds) + wave * (N / 4) + lane;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < KB * S::ND; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x16 &y = x[i / S::ND][i % S::ND];
                mine[(i * 4 + e) * 64] = f32x4{y[4 * e], y[4 * e + 1], y[4 * e + 2], y[4 * e + 3]};
            }
        __syncthreads();
        for (int i = wave; i < KB * S::ND; i += W) {
            const f32x4 *src = reinterpret_cast<const f32x4 *>(lds) + i * 4 * 64 + lane;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                f32x4 sum = src[e * 64];
#pragma unroll
                for (int w = 1; w < W; ++w) sum += src[w * (N / 4) + e * 64];
                const int key = 32 * (i / S::ND) + (lane & 31), col = 32 * (i % S::ND) + 8 * e + 4 * (lane >> 5);
                out.store<T>(sum * by, (key * at + col) * (int)sizeof(T), key < keys && col < d);
            }
        }
    }

    __device__ static void run(const SeqBwd &p, char *lds)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        BwdScale<T> sc;
        sc.find(p, lds);
        const int kvh = uniform((int)(blockIdx.x % p.Hkv));
        const int64_t t = (int)(blockIdx.x / p.Hkv);  // (earlier keys are seen by more rows: they start first)
        const int seq = uniform(seq_of_tile(p.seqs, t, 1, R, lane));
        if (seq < 0) return;
        const int row0 = uniform(p.seqs.start(seq)), n = uniform(p.seqs.length(seq));
        const int k0 = uniform((int)(t - tile0(p.seqs, seq, 1, R)) * R), Hq = p.Hkv * p.G;

        const Span ks((const T *)p.k + (row0 + k0) * p.ldk + kvh * p.d), vs((const T *)p.v + (row0 + k0) * p.ldv + kvh * p.d);
        frag kf[KB][S::NS], vf[KB][S::NS];
#pragma unroll
        for (int b = 0; b < KB; ++b) {
            const int kc = min(32 * b + (lane & 31), n - 1 - k0);
#pragma unroll
            for (int i = 0; i < S::NS; ++i) {
                const int col = (2 * i + (lane >> 5)) * S::V;
                u32x4 x = ks.load16((kc * (int)p.ldk + col) * (int)sizeof(T), col < p.d);
                __builtin_memcpy(&kf[b][i], &x, 16);
                x = vs.load16((kc * (int)p.ldv + col) * (int)sizeof(T), col < p.d);
                __builtin_memcpy(&vf[b][i], &x, 16);
            }
        }

        char *own = lds + wave * OWN;
        float *stats = reinterpret_cast<float *>(own + 4 * TILE);
        const int ldq = (int)p.ldq * (int)sizeof(T), ldg = Hq * p.d * (int)sizeof(T);
        Copy cq, cg;
        cq.init(ldq, p.d, 0, lane);
        cg.init(ldg, p.d, 0, lane);
        // The query tiles that see keys of this workgroup: of every head, first the
        // `part` ones that see some of them, then the others.
        const int from = p.causal ? k0 / 32 : 0, tiles = (n + 31) / 32 - from;
        const int part = p.causal ? min(KB, tiles) : 0;
        const int parts = p.G * part, all = p.G * tiles;
        float stat = 0.f;  // lanes 0..31: lse of a row of the next tile, 32..63: delta
        auto place = [&](int i, int &head, int &q0) {
            const int j = i < parts ? i : i - parts, each = i < parts ? part : tiles - part;
            const int g = j / each;
            head = uniform(kvh * p.G + g);
            q0 = uniform((from + (i < parts ? 0 : part) + j - g * each) * 32);
        };
        auto bring = [&](int i, int buf) {
            if (i >= all) return;
            int head, q0;
            place(i, head, q0);
            cq.tile((const T *)p.q + (row0 + q0) * p.ldq + head * p.d, n - q0, ldq, own + 2 * TILE * buf, 0);
            cg.tile((const T *)p.dout + ((int64_t)(row0 + q0) * Hq + head) * p.d, n - q0, ldg, own + 2 * TILE * buf + TILE, 0);
            const int r = q0 + (lane & 31);
            // (a row that is not there has weights of zero)
            stat = r < n ? (lane < 32 ? p.lse2 : p.delta)[(int64_t)head * p.seqs.total + row0 + r] : lane < 32 ? INFINITY : 0.f;
            if (lane < 32) stat -= BwdScale<T>::kP;
        };

        Grads x;
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt) x.dk[b][dt] = x.dv[b][dt] = f32x16{};
        const float scale = BwdScale<T>::kScaled ? sc.ds * 0x1p-14f : 1.f;
        bring(wave, 0);
        int i = wave, buf = 0;
#pragma unroll 1
        for (; i < parts; i += W, buf ^= 1) {
            int head, q0;
            place(i, head, q0);
            wave_arrived();
            stats[lane] = stat;
            bring(i + W, buf ^ 1);
            step<true>(own + 2 * TILE * buf, own + 2 * TILE * buf + TILE, stats, kf, vf, q0 - k0 - (lane & 31), 1 - q0, p.c, scale, x, lane);
        }
#pragma unroll 1
        for (; i < all; i += W, buf ^= 1) {
            wave_arrived();
            stats[lane] = stat;
            bring(i + W, buf ^ 1);
            step<false>(own + 2 * TILE * buf, own + 2 * TILE * buf + TILE, stats, kf, vf, 0, 0, p.c, scale, x, lane);
        }
        const int64_t out0 = ((int64_t)(row0 + k0) * p.Hkv + kvh) * p.d;
        add_up(lds, x.dk, Span((T *)p.dk + out0), n == 1 ? 0.f : p.c * kLn2 / sc.ds, p.Hkv * p.d, p.d, n - k0, wave, lane);
        add_up(lds, x.dv, Span((T *)p.dv + out0), BwdScale<T>::kScaled ? 0x1p-14f : 1.f, p.Hkv * p.d, p.d, n - k0, wave, lane);
    }
};

template <typename T, int D> __global__ __launch_bounds__(256, sizeof(T) == 4 && D > 64 ? 1 : 2) void seq_bwd_q(SeqBwd p)
{
    using U = SeqBwdQ<T, D>;
    __shared__ __attribute__((aligned(16))) char lds[U::LDS_BYTES];
    U::run(p, lds);
}

template <typename T, int D> __global__ __launch_bounds__((SeqBwdK<T, D>::NTH), 1) void seq_bwd_k(SeqBwd p)
{
    using U = SeqBwdK<T, D>;
    __shared__ __attribute__((aligned(16))) char lds[U::LDS_BYTES];
    U::run(p, lds);
}

}  // namespace ma
