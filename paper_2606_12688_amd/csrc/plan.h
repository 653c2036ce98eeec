// What the C-ABI's source files share: a plan and its device resources, the
// calling thread's error message, and the call that runs a plan's kernels.
#pragma once
#include <hip/hip_runtime.h>

#include <string>

#include "kernels.h"
#include "planner.h"

#define MSTAR_EXPORT extern "C" __attribute__((visibility("default")))

namespace mstar {

// Device-side resources of one plan: the device copy of the plan blob, its
// pinned staging copy, the events that order their reuse, and (for plans that
// run the few-row kernel beside the tile kernel) a side stream with its fork
// and join events.  Blocks are pooled per device: a destroyed plan returns its
// block and later plans take it back, so steady-state planning calls no
// hipMalloc / hipHostMalloc / hipFree (hipFree would also synchronize the
// device) and plan destruction makes no HIP call at all.
struct PlanBlock {
    int device = -1;
    size_t bytes = 0;          // capacity of dev and pinned
    void* dev = nullptr;
    void* pinned = nullptr;
    hipEvent_t uploaded = nullptr;  // after the last upload from `pinned`
    hipEvent_t last_use = nullptr;  // after the last fwd / kv_append enqueued outside graph capture
    bool uploaded_set = false, last_use_set = false;
    hipEvent_t ready = nullptr;     // the async planner's upload-done event
    hipStream_t side = nullptr;     // few-row kernel beside the tile kernel (default priority)
    hipEvent_t fork = nullptr, join = nullptr;
};

}  // namespace mstar

struct mstar_plan {
    mstar::HostPlan host;
    mstar::PlanBlock* blk = nullptr;  // device resources (NULL for a host-only plan)
    void* dev = nullptr;       // blk->dev
    size_t bytes = 0;
    size_t off_seqs = 0, off_row_hi = 0, off_tiles = 0, off_order = 0, off_few = 0, off_f32 = 0, off_merge = 0, off_append = 0, off_casc = 0, off_casc_rows = 0, off_casc_order = 0, off_err = 0;
    double plan_us = 0.0;
    // A plan with both tile and few-row items runs the few-row kernel on
    // blk->side beside the tile kernel: the caller's stream forks at blk->fork
    // and joins at blk->join before the merge.
    bool forked = false;
    bool from_planner = false;  // built by an async planner: blk->ready marks its upload
};

namespace mstar {

// Records `msg` as the calling thread's last error and returns `code`.
int fail(int code, const std::string& msg);
int hip_fail(hipError_t e, const char* what);

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

// The event that marks `plan`'s device blob as read by work enqueued on `s` (a
// later plan reusing the block waits for it): it goes with the call's last
// kernel.  NULL while `s` is being captured into a graph: a capture's replays
// are the caller's to finish before the plan is destroyed.
hipError_t use_event(const mstar_plan* plan, hipStream_t s, hipEvent_t* ev);

// The attention kernels of one kind of cache.
struct Launchers {
    hipError_t (*tiles)(const KArgs& a, int head_dim, hipStream_t s);
    hipError_t (*few)(const KArgs& a, int head_dim, int row_blocks, hipStream_t s);
    hipError_t (*cascade)(const KArgs& a, int head_dim, hipStream_t s);
    // NULL, or one launch for multi-row (or cascade) work and few-row items of one or two row blocks
    hipError_t (*mixed)(const KArgs& tile, const KArgs& few, bool cascade, int head_dim, int row_blocks, hipStream_t s);
};

// Checks the arguments and enqueues the plan's kernels (see mstar_attn_fwd_timed).
int run_fwd(const Launchers& kernels, const mstar_plan* plan, const void* q, const void* k_pages,
            const void* v_pages, const int32_t* block_table, void* out, float* lse, void* workspace,
            size_t workspace_bytes, hipStream_t stream, const hipEvent_t* events_before,
            const hipEvent_t* events_after);

// The same with the partials in the library's static device scratch (see mstar_attn_fwd_noalloc).
int run_fwd_noalloc(const Launchers& kernels, const mstar_plan* plan, const void* q, const void* k_pages,
                    const void* v_pages, const int32_t* block_table, void* out, float* lse, hipStream_t stream);

}  // namespace mstar
