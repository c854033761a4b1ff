// Host-side pieces of the exact attention over sequences and of the paged
// cache: what a call needs of the library's streams and workspaces
// (monarch_attn.hip), and the per-dtype dispatch (seq_fwd_*.hip, seq_bwd_*.hip).
#pragma once

#include <mutex>

#include "host_common.hpp"

namespace ma {
struct SeqFwd;
struct SeqBwd;
struct PagedPlan;
struct PagedWrite;
}  // namespace ma

namespace ma_host {

extern thread_local char g_err[512];  // what monarch_attn_last_error() returns

// Kernel kinds of the timing interface, after those of Kind.
enum SeqKind { kSeqFwd = 10, kSeqJoin = 11, kSeqStats = 12, kSeqBwd = 13, kSeqBwdJoin = 14, kPagedPlan = 15, kPagedWrite = 16 };

// The device, capture state and workspace of one call; `hold` keeps the
// workspace until the call's launches are enqueued.
struct CallScope {
    int dev = 0, num_cus = 0;
    bool capturing = false;
    char *ws = nullptr;
    std::unique_lock<std::mutex> hold;
};
// The current device.
int begin_call(CallScope &c);
// Its workspace, grown to `need` bytes (acquire_workspace).
int call_workspace(hipStream_t stream, size_t need, CallScope &c);
// Run the launches of one call, timed if timing is on, and check for launch errors.
int run_launches(hipStream_t stream, int (*f)(Launcher &, void *), void *arg);

bool ranges_overlap(const void *a, size_t na, const void *b, size_t nb);

// How a forward call runs.
struct SeqPlan {
    bool paged, split;
    int rows;       // packed rows a workgroup takes
    int64_t units;  // workgroups of one key head
};

// packed rows a workgroup takes: usually, and where sequences have few
template <typename T> constexpr int kSeqRows = sizeof(T) == 4 ? 64 : 128;
constexpr int kSeqFewRows = 32;
constexpr int kSeqThreads = 256;  // of a workgroup
inline int seq_rows(int32_t dtype) { return dtype == MA_F32 ? kSeqRows<float> : kSeqRows<__bf16>; }
// Workgroups of the split kernel that a compute unit holds: one where its K and V tiles take more
// than half of the LDS, 131 KB of 160 (fp32: few rows up to 64 columns, many rows past 64).
template <typename T> constexpr int seq_residents(int64_t d, bool few) { return sizeof(T) == 4 && few == (d <= 64) ? 1 : 2; }
inline int seq_residents(int32_t dtype, int64_t d, bool few) { return dtype == MA_F32 ? seq_residents<float>(d, few) : seq_residents<__bf16>(d, few); }
constexpr int kSeqBwdKeys = 64;  // keys a workgroup takes in the gradient

// rows of K and V that a workgroup writes into pages, of `chunks` times 16 bytes: about four chunks
// of each a thread
inline int paged_write_rows(int64_t chunks) { return (int)(chunks < 4 * kSeqThreads ? 4 * kSeqThreads / chunks : 1); }

template <typename T> int run_seq_fwd(Launcher &L, const ma::SeqFwd &p, const SeqPlan &how);
template <typename T> int run_seq_bwd(Launcher &L, const ma::SeqBwd &p);
int run_paged_plan(Launcher &L, const ma::PagedPlan &p);
int run_paged_write(Launcher &L, const ma::PagedWrite &p);

}  // namespace ma_host
