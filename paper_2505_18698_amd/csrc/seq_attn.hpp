// Exact attention over packed sequences and over paged caches.
//
// For every sequence, key head and group of query heads on it:
//   O_i = sum_j P_ij v_j,  P_ij = exp(s q_i.k_j - lse_i),  lse_i = log sum_j exp(s q_i.k_j),
// j over the keys that row i sees: the first vis(i) of the sequence.
#pragma once

#include "seq_tiles.hpp"

namespace ma {

// How a split call divides its work.  All row tiles of R rows in order, each with the key tiles (BN
// keys) of its sequence, are one line of `all` steps, which the workgroups share evenly: share w
// takes the steps from w all / shares on, in segments that lie in one row tile each.  So every
// workgroup ends at the same time whatever the contexts are, and starts once.  A row tile counts
// kBegin steps more than it has, for what its first copies, its rows and its masked key tiles take
// (measured in bf16 at 128 columns and used for all: 8 us to a step's 2 with 128 rows, 6 to 2.4
// with 32; without, the workgroups of 8 chunks of up to 512 tokens ended between 153 and 257 us).
//
// Of a share's segments only the first and the last can be parts of a row tile, and go to the
// partial results: where the share is the row tile's first one it is its last segment, number
// 2 w + 1 of share w, else its first, 2 w.
template <int R> constexpr int kBegin = R > 32 ? 4 : 2;
struct Line {
    int64_t all;       // steps
    int shares;        // workgroups that share them, four steps each at least
    int seq, tile;     // the row tile of the share's first step (seq = -1: none)
    int index;         // its number
    int64_t at;        // its first step
};

template <int R, int BN, int NTH>
__device__ inline Line find_share(const SeqFwd &p, int share, int max_keys, char *lds)
{
    int64_t *sh = reinterpret_cast<int64_t *>(lds);
    constexpr int W = NTH / 64;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    auto shape = [&](int s, int &rt, int &kt) {
        rt = s < p.seqs.B ? (int)(((int64_t)p.seqs.length(s) * p.G + R - 1) / R) : 0;
        const int kv = s < p.seqs.B ? max(0, min(p.kv_lens[s], max_keys)) : 0;
        kt = kBegin<R> + max(1, (kv + BN - 1) / BN);
    };
    int64_t sum = 0, tiles = 0;
    if (p.seqs.B > NTH) {  // (fewer: the sums below are those of all)
        for (int s = tid; s < p.seqs.B; s += NTH) {
            int rt, kt;
            shape(s, rt, kt);
            sum += (int64_t)rt * kt, tiles += rt;
        }
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x), tiles += __shfl_xor(tiles, x);
        if (lane == 0) sh[2 * wave] = sum, sh[2 * wave + 1] = tiles;
        __syncthreads();
        sum = tiles = 0;
        for (int i = 0; i < W; ++i) sum += sh[2 * i], tiles += sh[2 * i + 1];
        __syncthreads();
    }
    Line r{0, 0, -1, 0, 0, 0};
    int64_t want = 0, steps_before = 0, tiles_before = 0;
    for (int s0 = 0; s0 < p.seqs.B; s0 += NTH) {
        int rt, kt;
        shape(s0 + tid, rt, kt);
        int64_t t = rt, u = (int64_t)rt * kt;  // inclusive sums over the threads
        for (int x = 1; x < 64; x <<= 1) {
            const int64_t a = __shfl_up(t, x), b = __shfl_up(u, x);
            if (lane >= x) t += a, u += b;
        }
        if (lane == 63) sh[2 * wave] = t, sh[2 * wave + 1] = u;
        __syncthreads();
        int64_t at = 0, au = 0;
        for (int i = 0; i < W; ++i) {
            if (i < wave) t += sh[2 * i], u += sh[2 * i + 1];
            at += sh[2 * i], au += sh[2 * i + 1];
        }
        __syncthreads();
        if (s0 == 0) {
            if (p.seqs.B <= NTH) sum = au, tiles = at;
            // (row starts that decrease can make more row tiles than there is room for: those are
            // left out)
            if (blockIdx.x == 0 && tid == 0) p.parts[0].count = (int)min(tiles, (int64_t)p.tiles);
            r.all = sum, r.shares = (int)max((int64_t)1, min((int64_t)p.shares, sum / 4));
            if (share >= r.shares) return r;
            want = sum * share / r.shares;
        }
        const int64_t u0 = steps_before + u - (int64_t)rt * kt, k = want - u0;
        const bool mine = k >= 0 && k < (int64_t)rt * kt;  // one thread at most
        if (mine) {
            const int tile = (int)(k / kt);
            sh[0] = s0 + tid, sh[1] = tile, sh[2] = tiles_before + t - rt + tile, sh[3] = u0 + (int64_t)tile * kt;
        }
        if (some_thread<NTH>(mine, reinterpret_cast<int *>(lds + 64))) {
            r.seq = sh[2] < p.tiles ? (int)sh[0] : -1, r.tile = (int)sh[1], r.index = (int)sh[2], r.at = sh[3];
            break;
        }
        steps_before += au, tiles_before += at;
    }
    __syncthreads();
    return r;
}

// The share that step x of a line belongs to.
__device__ inline int share_of(int64_t x, int64_t all, int shares) { return (int)(((x + 1) * shares - 1) / all); }

// One workgroup of 4 waves per tile of R = 32 WR packed rows (token, head of
// the group) of one key head: the heads of a group read the same K and V, so
// they share the tile's copies.  With WR = 4 each wave owns 32 rows.  With WR = 1, for
// the few rows of single tokens, all waves copy, every wave takes one of the
// tile's 32-key parts, and the first joins them at the end.  WR = 2, in fp32: two
// row blocks by two 32-key parts (128 rows of 1000 keys are 54 us of a compute unit's fp32
// products, which one long sequence of a call then lasts).  Scores are formed
// transposed, S^T = K Q^T: a lane holds one query row's scores, so the softmax
// statistics and the rescaling are lane scalars with one exchange between the
// two lane halves, and the weights feed O^T = V^T P^T straight from registers.
//
// What bounds it.  Many rows: the products, 4 D operations a pair.  One causal sequence of 16384
// tokens, 16 heads on 4 of 128, bf16: 0.99 ms, 1.11 PFLOP/s (a library product of 8192^3 reaches
// 1.23), the matrix units busy in 61 % of the cycles, at the 1.76 GHz that the card's power leaves.
// There a tile's softmax (16 exponentials a lane and 32 x 32 block) runs on one of a SIMD's two
// waves beside the other's products, and no LDS bank conflict is left.  64 rows and key halves as
// in fp32 took 1.20 ms, 64 rows a wave 1.40 ms. Single tokens: the bytes of K and V.  64 requests
// of up to 8192 tokens, 32 heads on 8 of 128, bf16, 521 MB: 103 us, 5.1 TB/s; 2 of 131000, 1.07 GB:
// 190-197 us, 5.5 TB/s (a large copy reads and writes 4.9).
template <typename T, int D, int WR, bool PAGED, bool SPLIT> struct SeqAttn {
    using S = SeqTile<T, D>;
    using frag = typename S::frag;
    static constexpr int W = 4, NTH = 64 * W, R = 32 * WR;
    // Keys a tile.  Of few rows in 16-bit types, where the workgroup has a context
    // alone, 32 a wave.  Of few rows in fp32, whose products bound them as much as their bytes:
    // as many waves as the room lets work, four in one workgroup (D = 64: 152-162 us for the
    // contexts of 64 requests, 520 MB; 175 two in each of two, 197 one) or, past D = 64, one in
    // each of two (375 us, 1.04 GB; 432 two in one, 744 one in one).
    static constexpr int BN = WR != 1 ? 64 : S::kF32 ? (D <= 64 ? 128 : 32) : SPLIT ? 64 : 128;
    static constexpr int KT = WR == W ? BN / 32 : 1;       // 32-key parts that a wave takes
    static constexpr int KW = BN / 32 / KT;                // waves that share a tile's keys
    static_assert(WR * KW <= W, "rows and keys over the waves");
    static constexpr int TILE = BN * S::ROW;
    // Tiles that are there or on their way.  Short contexts of few rows are bound
    // by the latency of one tile after another: up to four, as the room allows.
    static constexpr int STAGES = WR != 1 || S::kF32 ? 2 : SPLIT ? (D <= 64 ? 4 : 2) : D <= 64 ? 3 : 2;
    static constexpr int LDS_BYTES = 2 * STAGES * TILE + 16;  // K and V
    using Copy = TileCopy<T, D, BN, W>;
    // A row's weights are taken relative to a reference that follows its running maximum only when
    // that has grown by more than 2^kSlack: the sums stay exact to fp32 (weights up to 2^kSlack),
    // and the output is rescaled a few times a row instead of once a tile.
    static constexpr float kSlack = 8.f;
    // fp16 holds 2^-24 to 65504: there all weights are taken times 2^kShift, up to 2^15, so that those
    // that become zero are below 2^-32 of the reference's (many keys below 2^-25 beside a large one
    // count in a long context: 2^17 of them were 0.4 % of the row).  The factor is in the sum too, and
    // leaves with it.
    static constexpr float kShift = std::is_same<T, _Float16>::value ? 7.f : 0.f;

    struct State {
        f32x16 o[S::ND];  // O^T: lane 32 h + c, row c, columns 32 dt + kRow32(r) + 4 h
        float ref, sum;
    };

    // One key tile.  MASK: some row of the tile sees only a part of it.  There
    // `fine` weights take part with twice the bits: rows of fewer keys than a tile, all of which
    // are in such tiles, have outputs as exact as the statistics.
    template <bool MASK>
    __device__ static void step(const char *kt, const char *vt, const frag *qf, int vis, int key0,
                                float c, bool fine, State &st, int lane)
    {
        f32x16 s[KT];
#pragma unroll
        for (int t = 0; t < KT; ++t) s[t] = f32x16{};
        constexpr int NK = KT * S::NS, NV = S::kF32 ? KT * 16 * S::ND : KT * 2 * S::ND, AHEAD = S::kF32 ? 2 : 4;
        FragStream<frag, S::kF32 ? NK : NK + NV, AHEAD> stream;
        auto load = [&](int u) {
            if constexpr (!S::kF32)
                if (u >= NK) return S::columns(vt + (u - NK) / S::ND * 16 * S::ROW, (u - NK) % S::ND, lane);
            return S::row_frag(kt + u / S::NS * 32 * S::ROW, u % S::NS, lane);
        };
        auto reads = [&](int u) { return u + AHEAD < NK ? 1 : S::kF32 || u + AHEAD >= NK + NV ? 0 : 2; };
        stream.start(load);
        __builtin_amdgcn_sched_group_barrier(kSchedDsRead, AHEAD, 0);
#pragma unroll
        for (int u = 0; u < NK; ++u) {
            stream.next(u, load, [&](const frag &x) {
                s[u / S::NS] = S::M::mma(x, qf[u % S::NS], s[u / S::NS]);
            });
            sched_step<(S::kF32 ? 4 : 1)>(reads(u));
        }
        Probs32<T> pf[KT];
        const int see = vis - key0 - 4 * (lane >> 5);
        float mx = -INFINITY;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                if (MASK && 32 * t + kRow32(r) >= see) s[t][r] = -INFINITY;
                mx = max_nan(mx, s[t][r]);
            }
        mx = wave_xor_max<32>(mx) * c;
        if (__any(mx > st.ref + kSlack)) {
            const float up = fmaxf(mx, st.ref);
            // (a row's first keys: all it has so far is zero, or infinities that take_foreign()
            // added)
            const float by = st.ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.ref - up);
            st.ref = up;
            st.sum *= by;
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt) st.o[dt] *= by;
        }
        const float ref = (st.ref == -INFINITY ? 0.f : st.ref) - kShift;
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r], c, -ref));
                sum += s[t][r];
            }
            pf[t].pack(s[t]);
        }
        st.sum += sum;
        if constexpr (S::kF32) {
            add_columns(vt, pf, st, lane);
        } else {
#pragma unroll
            for (int u = NK; u < NK + NV; ++u) {
                const int ks = (u - NK) / S::ND, dt = (u - NK) % S::ND;
                stream.next(u, load, [&](const frag &x) {
                    st.o[dt] = S::M::mma(x, pf[ks / 2].f[ks % 2], st.o[dt]);
                });
                sched_step<1>(reads(u));
            }
        }
        if constexpr (MASK && !S::kF32) {
            if (fine) {
#pragma unroll
                for (int t = 0; t < KT; ++t)
                    pf[t] = pf[t].rest(s[t]);
                add_columns(vt, pf, st, lane);
            }
        }
    }

    // O^T += V^T P^T of a tile.
    __device__ static void add_columns(const char *vt, const Probs32<T> *pf, State &st, int lane)
    {
#pragma unroll
        for (int k = 0; k < KT * (S::kF32 ? 16 : 2); ++k)
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt) {
                if constexpr (S::kF32) {
                    const float x = S::element(vt, 32 * (k / 16) + kRow32(k % 16) + 4 * (lane >> 5), dt, lane);
                    st.o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, pf[k / 16].s[k % 16], st.o[dt], 0, 0, 0);
                } else {
                    const frag x = S::columns(vt + k * 16 * S::ROW, dt, lane);
                    st.o[dt] = S::M::mma(x, pf[k / 2].f[k % 2], st.o[dt]);
                }
            }
    }

    // A value of V that is not finite meets weights of zero in the rows of a masked tile that do not
    // see it, where the product would make it NaN, and in the rows that do what `fine` adds to their
    // weights, of either sign.  So such values are looked for (`foreign`), added to the rows that see
    // them, and then taken for zero.
    __device__ static bool foreign(const char *vt)
    {
        bool bad = false;
        for (int i = threadIdx.x; i < TILE / 16; i += NTH) {
            T x[S::V];
            __builtin_memcpy(x, vt + i * 16, 16);
#pragma unroll
            for (int e = 0; e < S::V; ++e) bad |= !(fabsf((float)x[e]) < INFINITY);
        }
        return bad;
    }
    __device__ static void take_foreign(char *vt, int vis, int key0, bool mine, State &st, int lane)
    {
#pragma unroll 1
        for (int key = 0; key < (mine ? BN : 0); ++key) {
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int col = 32 * dt + kRow32(r) + 4 * (lane >> 5);
                    const float y = (float)*reinterpret_cast<const T *>(vt + key * S::ROW + (((col / S::V) ^ S::swz(key)) * 16) + col % S::V * (int)sizeof(T));
                    st.o[dt][r] += fabsf(y) < INFINITY || key0 + key >= vis ? 0.f : y;
                }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < TILE / (int)sizeof(T); i += NTH) {
            T &x = reinterpret_cast<T *>(vt)[i];
            if (!(fabsf((float)x) < INFINITY)) x = (T)0.f;
        }
        __syncthreads();
    }

    // The states of the waves that shared the tiles' keys, into the first one's.
    __device__ static void join_waves(char *lds, int wave, int lane, State &st)
    {
        constexpr int N = S::ND * 16 + 2;  // a lane's values of a row block
        static_assert((KW - 1) * WR * N * 256 <= 2 * STAGES * TILE, "the tiles' room holds them");
        float *mine = reinterpret_cast<float *>(lds) + (wave - WR) * N * 64 + lane;
        __syncthreads();
        if (wave >= WR && wave < KW * WR) {
            mine[(N - 2) * 64] = st.ref, mine[(N - 1) * 64] = st.sum;
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) mine[(dt * 16 + r) * 64] = st.o[dt][r];
        }
        __syncthreads();
        if (wave >= WR) return;
#pragma unroll
        for (int w = 1; w < KW; ++w) {
            const float *other = reinterpret_cast<float *>(lds) + ((w - 1) * WR + wave) * N * 64 + lane;
            const float ref = other[(N - 2) * 64], up = fmaxf(ref, st.ref), base = up == -INFINITY ? 0.f : up;
            // (a part without a key adds zeros, or infinities that take_foreign() added)
            const float a = st.ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(st.ref - base);
            const float b = ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - base);
            st.ref = up;
            st.sum = st.sum * a + other[(N - 1) * 64] * b;
#pragma unroll
            for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) st.o[dt][r] = st.o[dt][r] * a + other[(dt * 16 + r) * 64] * b;
        }
    }

    // The K and V rows that a wave copies.
    struct Rows {
        const T *k, *v;    // packed: the sequence's rows; paged: the key head's part of page 0
        const int *table;  // paged: the sequence's pages
        int kv;            // rows from this one on read as zero
        Copy ck, cv;
        int pages, page0;  // paged: lane i holds the sequence's page page0 + i

        // the pages of the tile from key0 on are among those that the lanes hold
        __device__ void look(const SeqFwd &p, int key0, int lane)
        {
            const int from = key0 >> p.page_log2, to = (key0 + BN - 1) >> p.page_log2;
            if (to - page0 < 64) return;
            page0 = from;
            pages = from + lane <= (kv - 1) >> p.page_log2 ? table[from + lane] : 0;
        }
        // the tile from key0 on
        __device__ void copy(const SeqFwd &p, int key0, char *kt, char *vt, int wave, int lane)
        {
            if constexpr (PAGED) {
                // A page holds the rows of a copy or several copies'.  Lane i finds
                // where copy i reads (in scalar registers, one copy after another, the
                // same took 140 instructions a tile, of 400 in all).
                look(p, key0, lane);
                const int ld = p.d * (int)sizeof(T);
                const int64_t each = (int64_t)(p.Hkv << p.page_log2) * ld;
                const int key = key0 + Copy::row(lane % Copy::COPIES, wave);
                const int pg = __shfl(pages, min((key >> p.page_log2) - page0, 63));
                const bool ok = (unsigned)pg < (unsigned)p.pages;
                const int64_t at = ok ? (int64_t)k + pg * each + (key & ((1 << p.page_log2) - 1)) * ld : (int64_t)&kNanRows;
                const int size = max(0, min(kv - key, Copy::RPC)) * ld, size_v = ok ? size : 0;
                const int64_t from_k = uniform((int64_t)v - (int64_t)k);
#pragma unroll
                for (int i = 0; i < Copy::COPIES; ++i) {
                    const int64_t a = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(at >> 32), i) << 32 |
                                                (uint32_t)__builtin_amdgcn_readlane((int)at, i));
                    ck.one(a, __builtin_amdgcn_readlane(size, i), kt, i, wave);
                    ck.one(a + from_k, __builtin_amdgcn_readlane(size_v, i), vt, i, wave);
                }
            } else {
                const int ldk = (int)p.ldk * (int)sizeof(T), ldv = (int)p.ldv * (int)sizeof(T);
                ck.tile(k + key0 * p.ldk, kv - key0, ldk, kt, wave);
                cv.tile(v + key0 * p.ldv, kv - key0, ldv, vt, wave);
            }
        }
    };

    __device__ static void run(const SeqFwd &p, char *lds)
    {
        const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6);
        const int kvh = uniform((int)(blockIdx.x % p.Hkv));
        const int max_keys = PAGED ? (int)min((int64_t)p.blocks << p.page_log2, (int64_t)0x7fffff00) : 0;  // (a tile behind the last one still has a number)
        if constexpr (SPLIT) {
            const int share = uniform((int)(blockIdx.x / p.Hkv));
            Line f = find_share<R, BN, NTH>(p, share, max_keys, lds);
            int seq = uniform(f.seq), tile = uniform(f.tile), index = uniform(f.index);
            if (seq < 0) return;
            const int shares = uniform(f.shares);
            const int64_t all = uniform(f.all), end = all * (share + 1) / shares;
            int64_t at = uniform(f.at), x = all * share / shares;
            while (x < end && index < p.tiles) {
                const int n = uniform(p.seqs.length(seq)), kv = uniform(max(0, min(p.kv_lens[seq], max_keys)));
                const int tiles = (int)(((int64_t)n * p.G + R - 1) / R), steps = max(1, (kv + BN - 1) / BN);
                if (tile >= tiles) {  // the next sequence
                    ++seq, tile = 0;
                    continue;
                }
                const int64_t begin = at + kBegin<R>, from = max(x, begin), stop = min(end, begin + steps);
                if (from < stop) {
                    const bool whole = from == begin && stop == begin + steps;
                    if (from == begin && kvh == 0 && tid == 0) {
                        const int last = share_of(begin + steps - 1, all, shares);
                        const int blind = kv == 0 ? n : p.causal ? max(0, n - kv) : 0;  // first tokens that see no key
                        p.parts[1 + index] = SeqTileParts{p.seqs.start(seq), tile * R, min(n * p.G - tile * R, R), share, last - share + 1, blind * p.G, {}};
                    }
                    segment(p, lds, tid, lane, wave, kvh, seq, tile, (int)(from - begin), (int)(stop - from), !whole,
                            (int64_t)(2 * share + (from == begin)) * p.Hkv + kvh, max_keys);
                    __syncthreads();  // the tiles' room is used again
                }
                at += kBegin<R> + steps, x = at, ++tile, ++index;
            }
        } else {
            if constexpr (!PAGED)
                if (p.clear) clear_outside<NTH>(p.seqs, p.out, (int64_t)p.Hkv * p.G * p.d * sizeof(T), blockIdx.x, gridDim.x);
            const int64_t t = p.tiles - 1 - (int)(blockIdx.x / p.Hkv);  // later rows see more keys: they start first
            const int seq = uniform(seq_of_tile(p.seqs, t, p.G, R, lane));
            if (seq < 0) return;
            segment(p, lds, tid, lane, wave, kvh, seq, uniform((int)(t - tile0(p.seqs, seq, p.G, R))), 0, 0x7fffffff, false, 0, max_keys);
        }
    }

    // Row tile `tile` of a sequence against `key_tiles` key tiles from key_tile0 on.
    // parts: the rows go to segment `unit` of the partial results.
    __device__ static __forceinline__ void segment(const SeqFwd &p, char *lds, int tid, int lane, int wave, int kvh, int seq, int tile,
                                                   int key_tile0, int key_tiles, bool parts, int64_t unit, int max_keys)
    {
        const int row0 = uniform(p.seqs.start(seq)), n = uniform(p.seqs.length(seq));
        const int kv = PAGED ? uniform(max(0, min(p.kv_lens[seq], max_keys))) : n;
        const int rows = n * p.G, r0 = tile * R;
        auto visible = [&](int r) {  // keys that packed row r sees (the last row stands for those behind it)
            const int64_t i = (int64_t)min(r, rows - 1) / p.G + (PAGED ? kv - n : 0) + 1;
            return p.causal ? (int)max((int64_t)0, min(i, (int64_t)kv)) : kv;
        };
        const int wr0 = r0 + wave % WR * 32;
        const int part = min(wave / WR, KW - 1);  // this wave's keys in a tile, in parts of 32
        const bool idle = wave >= WR * KW;
        const int see_most = uniform(visible(wr0 + 31));  // keys that some row of the wave sees
        const int see_all = uniform(visible(r0));  // keys that every row of the tile sees
        const int first = key_tile0 * BN;
        const int last = uniform((int)min((int64_t)visible(r0 + R - 1), key_tiles == 0x7fffffff ? (int64_t)0x7fffffff : (int64_t)(key_tile0 + key_tiles) * BN));

        // this lane's query rows; offsets of q and out from the tile's first token
        const int tok0 = r0 / p.G;
        const Span qs((const T *)p.q + (row0 + tok0) * p.ldq + (int64_t)kvh * p.G * p.d);
        frag qf[S::NS];
        const int row = wr0 + (lane & 31), r = min(row, rows - 1);
        const int vis = visible(r), tok = r / p.G - tok0, head = r % p.G;
#pragma unroll
        for (int i = 0; i < S::NS; ++i) {
            const int col = (2 * i + (lane >> 5)) * S::V;
            const u32x4 x = qs.load16((tok * (int)p.ldq + head * p.d + col) * (int)sizeof(T), col < p.d);
            __builtin_memcpy(&qf[i], &x, 16);
        }

        Rows src;
        src.kv = kv;
        if constexpr (PAGED) {
            src.k = (const T *)p.k + ((int64_t)kvh << p.page_log2) * p.d;
            src.v = (const T *)p.v + ((int64_t)kvh << p.page_log2) * p.d;
            src.table = p.table + (int64_t)seq * p.blocks;
            src.page0 = -0x10000, src.pages = 0;  // none yet
            src.ck.init(p.d * (int)sizeof(T), p.d, wave, lane);
        } else {
            const int ldk = (int)p.ldk * (int)sizeof(T), ldv = (int)p.ldv * (int)sizeof(T);
            src.k = (const T *)p.k + row0 * p.ldk + kvh * p.d;
            src.v = (const T *)p.v + row0 * p.ldv + kvh * p.d;
            src.ck.init(ldk, p.d, wave, lane);
            src.cv.init(ldv, p.d, wave, lane);
        }

        State st;
        st.ref = -INFINITY, st.sum = 0.f;
#pragma unroll
        for (int dt = 0; dt < S::ND; ++dt) st.o[dt] = f32x16{};
        // A tile arrives while the one or two before it are computed.  Two
        // loops, the tiles that every row sees whole and the others: one loop
        // with both kinds of step keeps the output registers twice.
        auto bring = [&](int key0, int buf) {
            if (key0 >= last) return;
            src.copy(p, key0, lds + 2 * TILE * buf, lds + 2 * TILE * buf + TILE, wave, lane);
        };
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) bring(first + i * BN, i);
        int key0 = first, buf = 0;
        auto arrive = [&] {
            if constexpr (STAGES == 2) {
                tile_barrier();
            } else {
                const int later = min(STAGES - 2, (last - 1 - key0) / BN);  // tiles on their way behind this one
                if (later >= 2) tile_barrier<4 * Copy::COPIES>();
                else if (later == 1) tile_barrier<2 * Copy::COPIES>();
                else tile_barrier();
            }
            bring(key0 + (STAGES - 1) * BN, buf == 0 ? STAGES - 1 : buf - 1);
        };
        auto next = [&] { key0 += BN, buf = buf == STAGES - 1 ? 0 : buf + 1; };
        // (a copy of the step for each buffer, whose LDS addresses are then constants: 1.01 ms for
        // 1.03 on the sequence of 16384 tokens; rows of 512 bytes and paged calls leave no
        // registers for it)
        constexpr int kCopies = !PAGED && D * sizeof(T) <= 256 ? STAGES : 1;
        const int whole = min(see_all, last) - BN;
#pragma unroll 1
        while (key0 <= whole) {
#pragma unroll
            for (int b = 0; b < kCopies; ++b) {
                if (key0 > whole) break;
                if (kCopies > 1) buf = b;
                arrive();
                char *kt = lds + 2 * TILE * (kCopies > 1 ? b : buf) + part * 32 * S::ROW;
                if (!idle) step<false>(kt, kt + TILE, qf, vis, key0 + 32 * part, p.c, p.rest != nullptr, st, lane);
                next();
            }
        }
#pragma unroll 1
        for (; key0 < last; next()) {
            arrive();
            char *vt = lds + 2 * TILE * buf + TILE;
            if ((p.causal || p.rest) && some_thread<NTH>(foreign(vt), reinterpret_cast<int *>(lds + 2 * STAGES * TILE)))
                take_foreign(vt, vis, key0, wave < WR, st, lane);
            if (key0 + 32 * part < see_most && !idle)
                step<true>(lds + 2 * TILE * buf + part * 32 * S::ROW, vt + part * 32 * S::ROW, qf, vis, key0 + 32 * part, p.c,
                           p.rest != nullptr, st, lane);
        }
        if constexpr (KW > 1) {
            join_waves(lds, wave, lane, st);
            if (wave >= WR) return;
        }

        const Span os((T *)p.out + ((row0 + tok0) * (int64_t)p.Hkv + kvh) * p.G * p.d);
        const float sum = wave_xor_sum<32>(st.sum);
        const bool none = vis <= first;  // no key to see
        const float inv = none ? 0.f : 1.f / sum;
        const float l2 = none ? -INFINITY : st.ref + (__builtin_amdgcn_logf(sum) - kShift);
        // A row has one owner: waves that only copied tiles have none. (They are here where no waves share
        // the keys: leaving as above cost 3 %, 64 tokens over up to 8192 in fp32, heads of 128.)
        const bool real = row < rows && wave < WR;
        if (SPLIT && parts) {
            const int64_t first_row = unit * R + wr0 - r0;
            const Span ps(p.part_o + first_row * D);
            // (scores of -infinity alone: a segment without a weight adds zeros to the row)
            store_row<float, S::ND>(ps, st.o, sum == 0.f ? 0.f : inv, (lane & 31) * D, D, real, lane);
            if (real && lane < 32) p.part_l[first_row + lane] = l2;
            return;
        }
        const int at = (tok * p.Hkv * p.G + head) * p.d;
        store_row<T, S::ND>(os, st.o, inv, at, p.d, real, lane);
        if constexpr (!S::kF32) {
            if (p.rest) {
                const Span es((T *)p.rest + ((row0 + tok0) * (int64_t)p.Hkv + kvh) * p.G * p.d);
#pragma unroll
                for (int dt = 0; dt < S::ND; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float x = st.o[dt][r] * inv;
                        st.o[dt][r] = x - (float)to_elem<T>(x);
                    }
                store_row<T, S::ND>(es, st.o, 1.f, at, p.d, real, lane);
            }
        }
        if (p.lse && real && lane < 32)
            p.lse[(int64_t)(kvh * p.G + head) * p.seqs.total + row0 + tok0 + tok] = l2 * kLn2;
    }
};

template <typename T, int D, int WR, bool PAGED, bool SPLIT>
__global__ __launch_bounds__(256, sizeof(T) == 4 && D > 64 && WR > 1 ? 1 : !PAGED && D * sizeof(T) <= 128 ? 3 : 2) void seq_attention(SeqFwd p)
{
    using U = SeqAttn<T, D, WR, PAGED, SPLIT>;
    __shared__ __attribute__((aligned(16))) char lds[U::LDS_BYTES];
    U::run(p, lds);
}

// Packed row `at` of a sequence if no segment has a weight of it: zero where it sees no key, else
// 0 / 0.
__device__ inline float without_weight(const SeqTileParts &f, int at) { return at < f.blind ? 0.f : NAN; }

// The segments of a split call's rows joined: O = sum_x w_x O_x / sum_x w_x, w_x = exp(lse_x). One
// workgroup per row tile and key head, and, of tiles of many rows, 8 rows, 32 threads a row (they
// have few segments); of 32-row tiles, `gridDim.y`-th of the rows, one at a time, 32 threads a
// segment and 8 segments at once.  5 us for single tokens, 13 us for 2786 rows of 32 heads, of
// which it reads 46 MB of segments.
template <typename T, int D, int R>
__global__ __launch_bounds__(256) void seq_join(SeqFwd p)
{
    constexpr int C = D / 32;  // columns a thread
    __shared__ float sh_o[8][D], sh_l[8];
    const int kvh = blockIdx.x % p.Hkv, tile = blockIdx.x / p.Hkv;
    const SeqTileParts f = p.parts[1 + tile];
    if (tile >= p.parts[0].count || f.count == 1) return;
    const int tid = threadIdx.x, g = tid / 32, c = tid % 32;
    // row r of the tile in its segment x (numbers as in find_share)
    const int64_t share = (int64_t)p.Hkv * R, base = 2 * f.first * share + kvh * R;
    auto part_row = [&](int x, int r) { return base + (x == 0 ? share : 2 * x * share) + r; };
    if constexpr (R > 32) {
        const int r = blockIdx.y * 8 + g;
        if (r >= f.rows) return;
        float mx = -INFINITY, sum = 0.f, o[C] = {};
        for (int x = 0; x < f.count; ++x) mx = max_nan(mx, p.part_l[part_row(x, r)]);
        const float ref = mx == -INFINITY ? 0.f : mx;
        for (int x = 0; x < f.count; ++x) {
            const float l = p.part_l[part_row(x, r)], w = l == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(l - ref);
            const float *src = p.part_o + part_row(x, r) * D + c * C;
            sum += w;
#pragma unroll
            for (int i = 0; i < C; ++i) o[i] = __builtin_fmaf(w, src[i], o[i]);
        }
        const int at = f.at + r;
        const float inv = mx == -INFINITY ? without_weight(f, at) : 1.f / sum;
        const int head = kvh * p.G + at % p.G;
        const int64_t row = f.row0 + at / p.G;
        T *out = (T *)p.out + (row * p.Hkv * p.G + head) * p.d + c * C;
#pragma unroll
        for (int i = 0; i < C; ++i)
            if (c * C + i < p.d) out[i] = to_elem<T>(o[i] * inv);
        if (p.lse && c == 0) p.lse[(int64_t)head * p.seqs.total + row] = mx == -INFINITY ? mx : (ref + __builtin_amdgcn_logf(sum)) * kLn2;
        return;
    }
    for (int r = blockIdx.y; r < f.rows; r += gridDim.y) {
        float mx = -INFINITY;
        for (int x = c; x < f.count; x += 32) mx = max_nan(mx, p.part_l[part_row(x, r)]);
#pragma unroll
        for (int x = 1; x < 32; x <<= 1) mx = max_nan(mx, __shfl_xor(mx, x));
        const float ref = mx == -INFINITY ? 0.f : mx;
        float sum = 0.f, o[C] = {};
#pragma unroll 4
        for (int x = g; x < f.count; x += 8) {
            const float l = p.part_l[part_row(x, r)];
            const float w = l == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(l - ref);  // (a segment of which this row sees nothing is zero)
            const float *src = p.part_o + part_row(x, r) * D + c * C;
            sum += w;
#pragma unroll
            for (int i = 0; i < C; ++i) o[i] = __builtin_fmaf(w, src[i], o[i]);
        }
#pragma unroll
        for (int i = 0; i < C; ++i) sh_o[g][c * C + i] = o[i];
        if (c == 0) sh_l[g] = sum;
        __syncthreads();
        if (tid < D) {
            float all = 0.f, y = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) all += sh_l[i], y += sh_o[i][tid];
            const int at = f.at + r;
            const int64_t row = f.row0 + at / p.G;
            const int head = kvh * p.G + at % p.G;
            if (tid < p.d) ((T *)p.out)[(row * p.Hkv * p.G + head) * p.d + tid] = to_elem<T>(mx == -INFINITY ? without_weight(f, at) : y / all);
            if (p.lse && tid == 0) p.lse[(int64_t)head * p.seqs.total + row] = mx == -INFINITY ? mx : (ref + __builtin_amdgcn_logf(all)) * kLn2;
        }
        __syncthreads();
    }
}

}  // namespace ma
