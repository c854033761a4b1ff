// Rotation of queries and keys by their positions, into other tensors or on the way into the paged
// cache.
//
// Pair i of a head, (a, b), at position t turns by the angle t f_i:
//   a' = a cos(t f_i) - b sin(t f_i),  b' = a sin(t f_i) + b cos(t f_i);
// the inverse turns by -t f_i, and is the gradient too. Pairs are the columns i and rot / 2 + i, or
// 2 i and 2 i + 1; columns from rot on stay.
#pragma once

#include "decoder_host.hpp"
#include "tiles.hpp"

namespace ma {

// (cos, sin) of t f.  The angle is formed in 64 bits, as turns, of which only the fraction counts:
// 53 bits hold a position of 31 and a frequency of 24 to 2^-22 of a turn at the worst, to 2^-37 at
// positions below 65536. The fraction then fits 32 bits.
__device__ inline float2 turn_of(int64_t t, float f)
{
    const double turns = (double)t * (double)f * 0.15915494309189533577;
    float2 r;
    sincospif(2.f * (float)(turns - rint(turns)), &r.y, &r.x);
    return r;
}

// The sequence that a row belongs to, or -1 (all lanes of a wave together).
__device__ inline int seq_of_row(const Seqs &q, int row, int lane)
{
    if (q.B == 0) return -1;
    int lo = 0, n = q.B;
    while (n > 1) {
        const int step = (n + 63) / 64;
        const int64_t at = (int64_t)lane * step;
        const int cnt = __popcll(__ballot(at < n && q.start(lo + (int)at) <= row));
        if (cnt == 0) return -1;
        lo += (cnt - 1) * step;
        n = min(step, n - (cnt - 1) * step);
    }
    return row >= q.start(lo) && row < q.start(lo + 1) ? lo : -1;
}

// A workgroup takes `rows` rows of all heads: first every row's angles, into LDS (one sine and cosine
// for all heads of a row), then V elements of both halves of a head a thread, the first ones on their way
// while the angles are formed.  What bounds it: bytes (bf16, 32 and 8 heads of 128: append of 15549 rows, 382 MB both
// ways, 77 us, 5.0 TB/s; of 64 rows 5.0 us, latency: the row's sequence, its length, then its sines).
template <typename T, int V, bool APPEND> __global__ __launch_bounds__(256) void rotate(Rotate p)
{
    typedef uint32_t vec __attribute__((ext_vector_type(V * sizeof(T) / 4)));
    __shared__ float2 turns[kRotateRows][64];
    __shared__ int64_t slot[kRotateRows];  // append: of the row, -1: none
    __shared__ int state[kRotateRows];     // 1: of a sequence
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int row0 = blockIdx.x * p.rows, rows = min(p.rows, p.seqs.total - row0);
    const int half = p.rot / 2, C = (p.d + 2 * V - 1) / (2 * V), turned = p.rot / (2 * V);
    const int H = p.Hq + (APPEND ? 2 : 1) * p.Hk;

    // this thread's item: chunk c of head h of row r, and the next ones 256 on
    int c = tid % C, h = tid / C % H, r = tid / C / H;
    const int step_c = 256 % C, step_h = 256 / C % H, step_r = 256 / C / H;
    vec a, b;
    // columns of the two vectors of an item
    auto columns = [&](int c, bool turns, int &x, int &y) {
        if (!turns) x = 2 * V * c, y = x + V;
        else if (p.interleaved) x = 2 * V * c, y = x + V;
        else x = V * c, y = half + x;
    };
    auto fetch = [&](int r, int h, int c) {
        if (r >= rows) return;
        const bool is_v = APPEND && h >= p.Hq + p.Hk;
        int x, y;
        columns(c, c < turned && !is_v, x, y);
        const int64_t row = row0 + r;
        const T *src = h < p.Hq ? (const T *)p.q + row * p.ldq + h * p.d
                       : is_v   ? (const T *)p.v + row * p.ldv + (h - p.Hq - p.Hk) * p.d
                                : (const T *)p.k + row * p.ldk + (h - p.Hq) * p.d;
        a = *(const vec *)(src + x);
        if (y < p.d) b = *(const vec *)(src + y);
    };
    fetch(r, h, c);

    for (int i = wave; i < rows; i += 4) {
        const int row = row0 + i, seq = seq_of_row(p.seqs, row, lane);
        if (lane == 0) {
            state[i] = seq >= 0;
            if constexpr (APPEND) {
                const int64_t s = p.slots[row];
                slot[i] = s >= 0 && s < (int64_t)p.pages << p.page_log2 && seq >= 0 ? s : -1;
            }
        }
        if (seq < 0) continue;
        const int64_t t = p.kv_lens ? (int64_t)p.kv_lens[seq] - (p.seqs.start(seq + 1) - row) : row - p.seqs.start(seq);
        if (lane < half) {
            float2 x = turn_of(t, p.inv_freq[lane]);
            if (p.inverse) x.y = -x.y;
            turns[i][lane] = x;
        }
    }
    __syncthreads();

    while (r < rows) {
        T x[V], y[V];
        __builtin_memcpy(x, &a, sizeof(a));
        __builtin_memcpy(y, &b, sizeof(b));
        const int r1 = r, h1 = h, c1 = c;
        c += step_c, h += step_h, r += step_r;
        if (c >= C) c -= C, ++h;
        if (h >= H) h -= H, ++r;
        fetch(r, h, c);

        const bool is_v = APPEND && h1 >= p.Hq + p.Hk, turns_it = c1 < turned && !is_v;
        if (turns_it) {
            auto turn = [](T &e, T &f, float2 t) {
                const float u = (float)e, v = (float)f;
                e = to_elem<T>(u * t.x - v * t.y);
                f = to_elem<T>(u * t.y + v * t.x);
            };
            const float2 *by = &turns[r1][c1 * V];
            if (p.interleaved) {
#pragma unroll
                for (int i = 0; i < V / 2; ++i) turn(x[2 * i], x[2 * i + 1], by[i]), turn(y[2 * i], y[2 * i + 1], by[V / 2 + i]);
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) turn(x[i], y[i], by[i]);
            }
        }
        const int64_t row = row0 + r1;
        T *dst;
        if (state[r1] == 0) {
            if (!p.clear) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = y[i] = (T)0.f;
        }
        if (h1 < p.Hq) {
            dst = (T *)p.q_out + (row * p.Hq + h1) * p.d;
        } else if constexpr (APPEND) {
            const int64_t s = slot[r1];
            if (s < 0) continue;
            const int head = h1 - p.Hq - (is_v ? p.Hk : 0), mask = (1 << p.page_log2) - 1;
            dst = (T *)(is_v ? p.v_out : p.k_out) + ((((s >> p.page_log2) * p.Hk + head) << p.page_log2) + (s & mask)) * p.d;
        } else {
            dst = (T *)p.k_out + (row * p.Hk + h1 - p.Hq) * p.d;
        }
        int to_x, to_y;
        columns(c1, turns_it, to_x, to_y);
        vec o;
        __builtin_memcpy(&o, x, sizeof(o));
        *(vec *)(dst + to_x) = o;
        __builtin_memcpy(&o, y, sizeof(o));
        if (to_y < p.d) *(vec *)(dst + to_y) = o;
    }
}

}  // namespace ma
