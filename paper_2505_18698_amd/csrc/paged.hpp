// The tables of a paged cache: what a step's lengths make of them, and the
// rows that go into it.
#pragma once

#include "../../include/monarch_attn.h"
#include "seq_params.hpp"
#include "tiles.hpp"

namespace ma {

constexpr int kPlanMaxB = MONARCH_ATTN_PLAN_MAX_B;

// Every workgroup forms the running sums over all requests in LDS (two integers a request,
// microseconds for thousands of them) and then takes its share of the new table entries and of the
// slots, one a thread, each finding its request by bisection. So the call is one launch without a
// wait between workgroups: the sums take less than a second launch would.  64 requests: 4.3 us; 512
// with 24045 new tokens: 6.7 us (10 with four slots a thread).  What bounds it is latency: the
// lengths, the sums, the free pages and the table are each read behind the one before.
static __global__ __launch_bounds__(256) void paged_plan(PagedPlan p)
{
    __shared__ int row_end[kPlanMaxB], page_end[kPlanMaxB];  // inclusive sums of new tokens and new pages
    __shared__ int64_t part[2][4];
    __shared__ int bad;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int page = 1 << p.page_log2;
    const int64_t room = min((int64_t)p.blocks << p.page_log2, (int64_t)0x7fffffff);  // tokens a request's row of the table holds
    const int free_first = p.free_in[0], free_count = p.free_in[1];  // (on their way while the sums are formed)
    if (tid == 0) bad = 0;
    __syncthreads();
    // of request s: the tokens before and after the step and the pages they take
    auto shape = [&](int s, int64_t &had, int64_t &have, int64_t &tokens, int &flags) {
        int64_t a = p.past[s], n = p.fresh[s];
        flags = a < 0 || n < 0 ? MA_PLAN_BAD_LENGTH : 0;
        a = max((int64_t)0, a), n = max((int64_t)0, n);
        if (a + n > room) flags |= MA_PLAN_TABLE_FULL;
        had = (min(a, room) + page - 1) >> p.page_log2;
        have = (min(a + n, room) + page - 1) >> p.page_log2;
        tokens = n;
    };
    int64_t rows = 0, pages = 0;
    for (int s0 = 0; s0 < p.B; s0 += 256) {
        int64_t had = 0, have = 0, n = 0;
        int flags = 0;
        if (s0 + tid < p.B) shape(s0 + tid, had, have, n, flags);
        if (flags) atomicOr(&bad, flags);
        int64_t r = n, g = have - had;
        for (int x = 1; x < 64; x <<= 1) {
            const int64_t a = __shfl_up(r, x), b = __shfl_up(g, x);
            if (lane >= x) r += a, g += b;
        }
        if (lane == 63) part[0][wave] = r, part[1][wave] = g;
        __syncthreads();
        int64_t ar = 0, ag = 0;
        for (int i = 0; i < 4; ++i) {
            if (i < wave) r += part[0][i], g += part[1][i];
            ar += part[0][i], ag += part[1][i];
        }
        __syncthreads();
        if (s0 + tid < p.B) {
            row_end[s0 + tid] = (int)min(rows + r, (int64_t)p.capacity);  // rows beyond the slots are left out
            page_end[s0 + tid] = (int)min(pages + g, (int64_t)0x7fffffff);
        }
        rows += ar, pages += ag;
    }
    __syncthreads();
    const int ring_len = max(1, p.ring_len);
    const int count = max(0, min(free_count, p.ring_len));
    int first = free_first % ring_len;
    if (first < 0) first += ring_len;
    auto taken_page = [&](int64_t e) { return e < count ? p.ring[(int)((first + e) % ring_len)] : -1; };
    auto request_of = [&](const int *end, int64_t x) {  // the first request whose sum exceeds x
        int lo = 0, hi = p.B - 1;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (end[mid] > x) hi = mid;
            else lo = mid + 1;
        }
        return lo;
    };

    const int64_t at = (int64_t)blockIdx.x * 256 + tid, step = (int64_t)gridDim.x * 256;
    for (int64_t s = at; s < p.B; s += step) {
        int64_t had, have, n;
        int flags;
        shape((int)s, had, have, n, flags);
        p.cu[s + 1] = row_end[s];
        p.kv_lens[s] = (int)min(max((int64_t)0, (int64_t)p.past[s]) + n, room);
    }
    for (int64_t e = at; e < min(pages, (int64_t)0x7fffffff); e += step) {
        const int s = request_of(page_end, e);
        int64_t had, have, n;
        int flags;
        shape(s, had, have, n, flags);
        const int64_t j = had + e - (page_end[s] - (have - had));
        if (j >= 0 && j < p.blocks) p.table[(int64_t)s * p.blocks + j] = taken_page(e);
    }
    const int end = p.B > 0 ? row_end[p.B - 1] : 0;
    for (int64_t r = at; r < p.capacity; r += step) {
        int64_t slot = -1;
        if (r < end) {
            const int s = request_of(row_end, r);
            int64_t had, have, n;
            int flags;
            shape(s, had, have, n, flags);
            const int64_t pos = max((int64_t)0, (int64_t)p.past[s]) + r - (s ? row_end[s - 1] : 0);
            const int64_t j = pos >> p.page_log2;
            if (j < p.blocks) {
                const int pg = j < had ? p.table[(int64_t)s * p.blocks + j] : taken_page(page_end[s] - (have - had) + j - had);
                if (pg >= 0) slot = ((int64_t)pg << p.page_log2) + (pos & (page - 1));
            }
        }
        p.slots[r] = slot;
    }
    if (blockIdx.x == 0 && tid == 0) {
        const int used = (int)min(pages, (int64_t)count);
        p.cu[0] = 0;
        p.free_out[0] = (int)(((int64_t)first + used) % ring_len);
        p.free_out[1] = count - used;
        p.status[0] = bad | (pages > count ? MA_PLAN_NO_PAGES : 0) | (rows > p.capacity ? MA_PLAN_NO_SLOTS : 0);
    }
}

// Row r of k and v to slot slots[r], 16 bytes a thread.  A row whose slot is not
// in the cache is not written.  Bound by its bytes: 18951 rows of 8 heads of 128 in bf16,
// 155 MB: 28 us, 5.5 TB/s.
static __global__ __launch_bounds__(256) void paged_write(PagedWrite p, int per)
{
    const int chunks = p.Hkv * p.d * p.size / 16, head = p.d * p.size / 16;
    const int64_t r0 = (int64_t)blockIdx.x * per;
    const int n = (int)min((int64_t)per, p.rows - r0) * chunks;
    const int64_t slots = (int64_t)p.pages << p.page_log2;
#pragma unroll 4
    for (int i = threadIdx.x; i < n; i += 256) {
        const int r = i / chunks, c = i - r * chunks, h = c / head;
        const int64_t slot = p.slots[r0 + r];
        if (slot < 0 || slot >= slots) continue;
        const u32x4 a = *((const u32x4 *)((const char *)p.k + (r0 + r) * p.ldk * p.size) + c);
        const u32x4 b = *((const u32x4 *)((const char *)p.v + (r0 + r) * p.ldv * p.size) + c);
        const int64_t to = ((((slot >> p.page_log2) * p.Hkv + h) << p.page_log2) + (slot & ((1 << p.page_log2) - 1))) * head + c - h * head;
        ((u32x4 *)p.k_pages)[to] = a;
        ((u32x4 *)p.v_pages)[to] = b;
    }
}

}  // namespace ma
