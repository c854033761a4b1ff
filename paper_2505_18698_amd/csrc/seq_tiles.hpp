// Tiles of the exact attention over packed and paged sequences: 32 x 32
// products whose left operand comes from swizzled row-major LDS tiles, the
// copies that fill those tiles from global memory, and the search for the
// sequence that a tile of packed rows belongs to.
#pragma once

#include "seq_params.hpp"
#include "tiles.hpp"

namespace ma {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef const __attribute__((address_space(1))) void *global_ptr;
typedef __attribute__((address_space(3))) void *lds_ptr;

// One 32 x 32 step: 16 elements of the contraction in 16-bit types; 8 in fp32,
// as four instructions of depth 2, operand slot (half, i) being element 4 half + i.
template <typename T> struct Mma32;
template <> struct Mma32<__bf16> {
    using frag = bf16x8;
    __device__ static f32x16 mma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mma32<_Float16> {
    using frag = f16x8;
    __device__ static f32x16 mma(frag a, frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Mma32<float> {
    using frag = f32x4;
    __device__ static f32x16 mma(frag a, frag b, f32x16 c)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};

// Result layout of a 32 x 32 step: lane 32 h + c holds column c, rows kRow32(r) + 4 h, r = 0..15.
__device__ constexpr int kRow32(int r) { return 8 * (r / 4) + r % 4; }

// A row-major LDS tile of rows of D elements in 16-byte chunks, PC chunks a
// row.  Chunk c of row r lies at c ^ swz(r).  The LDS has 64 banks of 4 bytes,
// 16 chunks: a pass of a 16-byte read takes one column of 16 rows, all different
// modulo 16; of a transposing read, 4 columns of 4 consecutive rows; of a
// 4-byte read, 8 columns of the rows r and r + 4.  swz puts each on 16 different
// chunks of banks.  (With 8 different ones, c ^ f(r % 8), the counters showed 4 cycles more
// for each 16-byte read and 2 for each transposing one.)
template <typename T, int D> struct SeqTile {
    static constexpr int V = 16 / (int)sizeof(T);           // elements a chunk
    static constexpr int PC = D * (int)sizeof(T) <= 128 ? 8 : D * (int)sizeof(T) <= 256 ? 16 : 32;
    static constexpr int ROW = PC * 16;                     // bytes a row
    static constexpr int NS = D / (2 * V);                  // steps of a product over D
    static constexpr int ND = D / 32;                       // 32-wide tiles of D
    static constexpr bool kF32 = sizeof(T) == 4;
    using M = Mma32<T>;
    using frag = typename M::frag;

    __device__ static int swz(int row)
    {
        if constexpr (kF32) return ((row >> 2) & 1) << 3 | (row & 3) << 1 | ((row >> 3) & 1);
        else if constexpr (PC == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);  // (two rows to the 64 banks)
        else return (row & 3) << 2 | ((row >> 2) & 3);
    }

    // Operand fragment of the rows: lane 32 h + c holds chunk 2 st + h of row c of the 32 from
    // `rows` on.
    __device__ static frag row_frag(const char *rows, int st, int lane)
    {
        return *reinterpret_cast<const frag *>(rows + (lane & 31) * ROW + ((2 * st) ^ (lane >> 5) ^ swz(lane & 15)) * 16);
    }

    // Operand fragment X^T: lane 32 h + c holds column 32 dt + c of the rows
    // 4 h + 0..3 and 8 + 4 h + 0..3 of the 16 rows from `rows` on (16-bit types).
    __device__ static frag columns(const char *rows, int dt, int lane)
    {
        const int j = lane & 15, r = 4 * (lane >> 5) + (j >> 2);
        const int chunk = 4 * dt + 2 * ((lane >> 4) & 1) + ((j >> 1) & 1);
        const char *x = rows + r * ROW + (j & 1) * 8;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(x + ((chunk ^ swz(r)) * 16)));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(x + 8 * ROW + ((chunk ^ swz(r + 8)) * 16)));
        frag f;
        __builtin_memcpy(&f, &lo, 8);
        __builtin_memcpy((char *)&f + 8, &hi, 8);
        return f;
    }

    // Element (row, 32 dt + lane % 32) of the tile (fp32).
    __device__ static float element(const char *tile, int row, int dt, int lane)
    {
        const int c = lane & 31;
        return *reinterpret_cast<const float *>(tile + row * ROW + (((8 * dt + (c >> 2)) ^ swz(row)) * 16) + (c & 3) * 4);
    }
};

// Two values per row of a 32 x 32 result, each as a product of its own: a lane of the left operand
// holds its row's x in three slots, as bf16 values whose sum is x to 2^-24, and y in three others;
// the right operand holds ones in either's. So they reach all results of the row without passing
// through LDS.  (fp32: x and y in the two slots.)
template <typename T> struct RowTerms {
    bf16x8 a;
    // x and y finite: an infinity would meet itself in the second value
    __device__ inline void set(float x, float y, int lane)
    {
        a = bf16x8{};
        if (lane < 32) {
            float z[2] = {x, y};
#pragma unroll
            for (int i = 0; i < 6; ++i) {
                a[i] = (__bf16)z[i / 3];
                z[i / 3] -= (float)a[i];
            }
        }
    }
    template <int I> __device__ inline f32x16 add(f32x16 c, int lane) const
    {
        const uint32_t one = lane < 32 ? 0x3f803f80u : 0u;  // two bf16 ones
        const u32x4 ones = I == 0 ? u32x4{one, one & 0xffffu, 0u, 0u} : u32x4{0u, one & 0xffff0000u, one, 0u};
        bf16x8 b;
        __builtin_memcpy(&b, &ones, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
    }
};
template <> struct RowTerms<float> {
    float a;
    __device__ inline void set(float x, float y, int lane) { a = lane < 32 ? x : y; }
    template <int I> __device__ inline f32x16 add(f32x16 c, int lane) const
    {
        return __builtin_amdgcn_mfma_f32_32x32x2f32(a, lane / 32 == I ? 1.f : 0.f, c, 0, 0, 0);
    }
};

// The 32 x 32 result `s` as the right operand of products that contract over
// its rows: two fragments of 16 rows in 16-bit types, the values themselves in fp32.
// (So the weights, and in the gradient dS, are rounded to the element type, the one rounding besides that of the
// outputs: the matrix instructions take no wider operand, and a second product with what rounding left, as masked tiles
// have it, would double those of V. In bf16 outputs and gradients of cross attention are 2.2e-3 to 2.4e-3 from 64 bits, 1.7e-3
// of which the outputs' own rounding is; in fp16 2.8e-4 and 2.0e-4.)
template <typename T> struct Probs32 {
    typename Mma32<T>::frag f[2];
    __device__ inline void pack(f32x16 s)
    {
#pragma unroll
        for (int r = 0; r < 16; ++r) f[r / 8][r % 8] = to_elem<T>(s[r]);
    }
    // what pack(s) left of s
    __device__ inline Probs32 rest(f32x16 s) const
    {
        Probs32 x;
#pragma unroll
        for (int r = 0; r < 16; ++r) x.f[r / 8][r % 8] = to_elem<T>(s[r] - (float)f[r / 8][r % 8]);
        return x;
    }
};
template <> struct Probs32<float> {
    f32x16 s;
    __device__ inline void pack(f32x16 x) { s = x; }
};

// A step's fragments, in the order in which its products use them, read from
// LDS AHEAD of them in front of their use: a read takes as long as several
// products, and left to itself the compiler waits for each read in front of its
// own.  `load(u)`: fragment u of N; every loop over them is unrolled.
enum SchedGroup { kSchedMfma = 0x8, kSchedDsRead = 0x100 };
template <typename Frag, int N, int AHEAD> struct FragStream {
    Frag f[AHEAD];
    template <typename Load> __device__ __forceinline__ void start(Load &&load)
    {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) f[u] = load(u);
    }
    // Fragment u for the products `use`, and the read of one that comes later.
    template <typename Load, typename Use> __device__ __forceinline__ void next(int u, Load &&load, Use &&use)
    {
        use(f[u % AHEAD]);
        if (u + AHEAD < N) f[u % AHEAD] = load(u + AHEAD);
    }
};
// The order of one product (PRODUCTS instructions) and the `reads` (0 to 2) behind it.
template <int PRODUCTS> __device__ __forceinline__ void sched_step(int reads)
{
    __builtin_amdgcn_sched_group_barrier(kSchedMfma, PRODUCTS, 0);
    if (reads == 1) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 1, 0);
    if (reads == 2) __builtin_amdgcn_sched_group_barrier(kSchedDsRead, 2, 0);
}

// One row (lane % 32) of X^T, held as 32 x 32 results, times `by`, to element `at`
// behind a base: 16 bytes a store.  In 16-bit types a lane holds 8 bytes of every 16, its
// partner in the other half of the wave the rest; of two such pairs each takes one.
template <typename O, int ND>
__device__ inline void store_row(const Span &s, const f32x16 *x, float by, int at, int d, bool real, int lane)
{
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) {
        if constexpr (sizeof(O) == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int col = 32 * dt + 8 * e + 4 * (lane >> 5);
                s.store<O>(f32x4{x[dt][4 * e] * by, x[dt][4 * e + 1] * by, x[dt][4 * e + 2] * by, x[dt][4 * e + 3] * by},
                           (at + col) * 4, real && col < d);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                uint32_t w[4];  // columns 8 e + 4 h.. and 8 (e + 1) + 4 h.. of the row, two dwords each
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = 4 * (e + i / 2) + 2 * (i % 2);
                    O v[2] = {to_elem<O>(x[dt][r] * by), to_elem<O>(x[dt][r + 1] * by)};
                    __builtin_memcpy(&w[i], v, 4);
                }
                const auto lo = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
                const auto hi = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
                const int col = 32 * dt + 8 * (e + (lane >> 5));
                __builtin_amdgcn_raw_buffer_store_b128(u32x4{lo[0], hi[0], lo[1], hi[1]}, s.r, Span::at((at + col) * 2, real && col < d), 0, 0);
            }
        }
    }
}

// A value that all lanes of the wave share, in a scalar register: the address of a copy has to be
// there.
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)x), hi = __builtin_amdgcn_readfirstlane((int)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// What a page outside the cache reads as: NaN in every type.
static __device__ __align__(16) const struct NanRows { uint32_t x[256]; } kNanRows = [] {
    NanRows n{};
    for (uint32_t &x : n.x) x = 0x7fff7fffu;
    return n;
}();

// The copies global -> LDS that fill a tile of BN rows: copy i of wave w fills
// the RPC rows from (i NW + w) RPC on, 16 bytes a lane, from rows `ld` bytes
// apart that start at a uniform address.  Rows past the `valid` ones and
// columns past d read as zero, by the range check of the buffer access.
template <typename T, int D, int BN, int NW> struct TileCopy {
    using S = SeqTile<T, D>;
    static constexpr int RPC = 64 / S::PC, COPIES = BN / RPC / NW;
    static constexpr int VAR = NW * RPC >= 16 ? 1 : 16 / (NW * RPC);  // copies after which a lane's column comes again
    static_assert(COPIES * NW * RPC == BN && COPIES % VAR == 0, "whole copies");
    int off[VAR];  // this lane's chunk, from the first row of the copy

    __device__ void init(int ld, int d, int wave, int lane)
    {
#pragma unroll
        for (int i = 0; i < VAR; ++i) {
            const int r = lane / S::PC, col = ((lane % S::PC) ^ S::swz((row(i, wave) + r) & 15)) * S::V;
            off[i] = col < d ? r * ld + col * (int)sizeof(T) : (int)0x80000000;
        }
    }
    // first row of copy i in the tile
    __device__ static int row(int i, int wave) { return (i * NW + wave) * RPC; }
    // the descriptor of a buffer access that reads zero behind `valid` rows
    __device__ static u32x4 source(const void *rows, int valid, int ld)
    {
        const int64_t at = uniform((int64_t)rows);
        return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)uniform(max(0, min(valid, BN)) * ld), (uint32_t)Span::kDefault};
    }
    // The copy itself, in assembly: behind the builtin the compiler waits for it
    // before every later LDS read, those of the other tiles among them, so that
    // a tile would not arrive while another is computed.  The instruction writes LDS and
    // no register; tile_barrier() waits for it.
    // (The compiler does not see into it either: the five wait states are
    // those between a vector write of a scalar register and its use here.)
    __device__ static void copy(u32x4 r, int off, char *tile, int i, int wave)
    {
        const int to = (int)(uintptr_t)(lds_ptr)tile + row(i, wave) * S::ROW;
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds"
                     :: "v"(off), "s"(r), "s"(uniform(to)) : "memory", "m0");
    }
    // copy i alone, from its own first row, of which `size` bytes can be read
    __device__ void one(int64_t rows, int size, char *to, int i, int wave) const
    {
        copy(u32x4{(uint32_t)rows, (uint32_t)(rows >> 32) & 0xffffu, (uint32_t)size, (uint32_t)Span::kDefault}, off[i % VAR], to, i, wave);
    }
    // the whole tile from its first row
    __device__ void tile(const void *rows, int valid, int ld, char *to, int wave) const
    {
        const u32x4 r = source(rows, valid, ld);
#pragma unroll
        for (int i = 0; i < COPIES; ++i) copy(r, off[i % VAR] + row(i, wave) * ld, to, i, wave);
    }
};

// All but the last LATER copies of this wave (and all its LDS accesses) are done.
// (The wait is the builtin, not assembly, so that the compiler knows of it: it
// would wait again in front of the first use of what was loaded before the loop, in
// every iteration, and there for copies that it does not know of.)
template <int LATER = 0> __device__ inline void copies_arrived()
{
    static_assert(LATER < 64, "6 bits");
    __builtin_amdgcn_s_waitcnt((LATER & 15) | 0x70 | (LATER >> 4) << 14);  // vmcnt(LATER) lgkmcnt(0)
}

// The same, and every wave of the workgroup is here.
template <int LATER = 0> __device__ inline void tile_barrier()
{
    copies_arrived<LATER>();
    asm volatile("s_barrier" ::: "memory");
}

// Whether `x` holds on some thread of a workgroup of NTH (`shared`: NTH / 64 integers of LDS).
template <int NTH> __device__ inline bool some_thread(bool x, int *shared)
{
    const int tid = threadIdx.x;
    const bool mine = __any(x);
    if (tid % 64 == 0) shared[tid / 64] = mine;
    __syncthreads();
    int any = 0;
#pragma unroll
    for (int i = 0; i < NTH / 64; ++i) any |= shared[i];
    __syncthreads();
    return uniform(any) != 0;
}

// ---- sequences ----

// Zeros in the rows of no sequence of x, rows of `bytes` bytes (a multiple of
// 16): the share of workgroup `block` of `blocks`.
template <int NTH> __device__ inline void clear_outside(const Seqs &q, void *x, int64_t bytes, int64_t block, int64_t blocks)
{
    const int first = q.start(0), last = max(first, q.start(q.B));
    const int64_t before = first * bytes / 16, all = before + (q.total - last) * bytes / 16;
    for (int64_t i = block * NTH + threadIdx.x; i < all; i += blocks * NTH)
        reinterpret_cast<u32x4 *>(x)[i < before ? i : i - before + last * bytes / 16] = u32x4{0u, 0u, 0u, 0u};
}

// Sequence s holds tiles tile0(s) .. tile0(s) + ceil(rows / R) - 1 of R packed
// rows, tile0(s) = floor(first row / R) + s: with ceil(n / R) <= floor((x + n) / R)
// - floor(x / R) + 1 the ranges of two sequences never meet, and no prefix sum
// over the sequences is needed.  G: packed rows a token.
__device__ inline int64_t tile0(const Seqs &q, int s, int G, int R) { return (int64_t)q.start(s) * G / R + s; }

// The sequence of tile t (all lanes of a wave together; 64 candidates a step),
// or -1 where t is no tile of any.
__device__ inline int seq_of_tile(const Seqs &q, int64_t t, int G, int R, int lane)
{
    if (q.B == 0) return -1;
    int lo = 0, n = q.B;
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int64_t at = (int64_t)lane * step;
        const int cnt = __popcll(__ballot(at < n && tile0(q, lo + (int)at, G, R) <= t));
        if (cnt == 0) return -1;
        lo += (cnt - 1) * step;
        n = min(step, n - (cnt - 1) * step);
    }
    const int64_t k = t - tile0(q, lo, G, R);
    return k >= 0 && k * R < (int64_t)q.length(lo) * G ? lo : -1;
}

}  // namespace ma
