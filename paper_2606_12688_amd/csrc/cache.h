// Launch interface of the operators on paged caches (mstar_cache.h).
#pragma once
#include "kernels.h"
#include "mstar_cache.h"

namespace mstar {

struct Append4Args {
    const SeqInfo* seqs;
    const WorkItem* items;  // rows row0 .. row0 + nrows - 1 of request seq, at positions [k_begin, k_end)
    const void* k_new;      // [total_q][hkv][head_dim] bf16
    const void* v_new;
    const int32_t* bt;
    void* k;                // 4-bit pools
    void* v;
    int32_t* err;           // sticky device error word
    int32_t n_items;
    int32_t hkv, bt_stride, num_pages;
    hipEvent_t done;  // host side: NULL, or an event that completes with the kernel (not under capture)
};

struct Unpack4Args {
    const void* k;  // 4-bit pools
    const void* v;
    const int32_t* ids;
    void* k_out;    // [n_ids][16][hkv][head_dim] bf16
    void* v_out;
    int32_t n_ids, hkv, num_pages;
    int32_t n_wgs;    // set by the launch
    hipEvent_t done;  // NULL
};

struct TablesArgs {
    const SeqInfo* seqs;
    const WorkItem* items;  // as for the append
    const int32_t* free_pages;
    int32_t* bt;
    int64_t* slots;         // NULL: no slot map
    int32_t* err;
    int32_t n_items;
    int32_t bt_stride, num_pages;
    hipEvent_t done;
};

hipError_t launch_append4(const Append4Args& a, int head_dim, hipStream_t s);
hipError_t launch_unpack4(const Unpack4Args& a, int head_dim, hipStream_t s);
hipError_t launch_tables(const TablesArgs& a, hipStream_t s);

// Attention over a 4-bit cache: k and v of KArgs are 4-bit pools.
hipError_t launch_tiles4(const KArgs& a, int head_dim, hipStream_t s);
hipError_t launch_cascade4(const KArgs& a, int head_dim, hipStream_t s);
// Multi-row (or cascade) work and few-row items of one or two row blocks in one
// launch; tile.done goes with it.
hipError_t launch_mixed4(const KArgs& tile, const KArgs& few, bool cascade, int head_dim, int row_blocks, hipStream_t s);
hipError_t launch_few4(const KArgs& a, int head_dim, int row_blocks, hipStream_t s);

}  // namespace mstar
