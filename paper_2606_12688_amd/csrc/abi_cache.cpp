// C-ABI of the operators on paged caches (mstar_cache.h): argument checks and
// launches.  As in abi.cpp, nothing here throws across the boundary.
#include <hip/hip_runtime.h>

#include "cache.h"
#include "plan.h"

using mstar::aligned;
using mstar::fail;
using mstar::hip_fail;

namespace {

// What every call with a plan needs: a plan with device buffers, on the current
// device (its buffers, and with them the caller's tensors, live there).
int check_plan(const mstar_plan* plan) {
    if (!plan) return fail(MSTAR_ERR_INVALID_ARG, "plan is NULL");
    if (!plan->dev) return fail(MSTAR_ERR_INVALID_ARG, "plan was built host-only");
    int dev = 0;
    const hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return hip_fail(e, "hipGetDevice");
    if (dev != plan->blk->device) return fail(MSTAR_ERR_INVALID_ARG, "the plan was built on another device");
    return MSTAR_OK;
}

int check_plan4(const mstar_plan* plan) {
    const int rc = check_plan(plan);
    if (rc != MSTAR_OK) return rc;
    if (plan->host.params.dtype != MSTAR_DTYPE_BF16)
        return fail(MSTAR_ERR_UNSUPPORTED, "a 4-bit cache needs a plan of the bf16 dtype");
    return MSTAR_OK;
}

constexpr mstar::Launchers kKernels4 = {mstar::launch_tiles4, mstar::launch_few4, mstar::launch_cascade4,
                                        mstar::launch_mixed4};

template <typename T>
T* at(const mstar_plan* plan, size_t off) {
    return reinterpret_cast<T*>(static_cast<unsigned char*>(plan->dev) + off);
}

}  // namespace

MSTAR_EXPORT int mstar_kv4_append(const mstar_plan_t* plan, const void* k_new, const void* v_new,
                                  const int32_t* block_table, void* k_pages, void* v_pages, hipStream_t stream) {
    const int rc = check_plan4(plan);
    if (rc != MSTAR_OK) return rc;
    const mstar::HostPlan& h = plan->host;
    if (h.appends.empty()) return MSTAR_OK;
    if (!k_new || !v_new || !block_table || !k_pages || !v_pages)
        return fail(MSTAR_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) ||
        !aligned(block_table, 4))
        return fail(MSTAR_ERR_INVALID_ARG, "k_new/v_new/k_pages/v_pages must be 16-byte aligned");
    mstar::Append4Args a{};
    a.seqs = at<const mstar::SeqInfo>(plan, plan->off_seqs);
    a.items = at<const mstar::WorkItem>(plan, plan->off_append);
    a.k_new = k_new;
    a.v_new = v_new;
    a.bt = block_table;
    a.k = k_pages;
    a.v = v_pages;
    a.err = at<int32_t>(plan, plan->off_err);
    a.n_items = (int32_t)h.appends.size();
    a.hkv = h.params.num_kv_heads;
    a.bt_stride = h.params.max_blocks_per_seq;
    a.num_pages = h.params.num_pages;
    hipError_t e = mstar::use_event(plan, stream, &a.done);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if ((e = mstar::launch_append4(a, h.params.head_dim, stream)) != hipSuccess)
        return hip_fail(e, "4-bit append kernel launch");
    if (a.done) plan->blk->last_use_set = true;
    return MSTAR_OK;
}

MSTAR_EXPORT int mstar_kv4_fwd(const mstar_plan_t* plan, const void* q, const void* k_pages, const void* v_pages,
                               const int32_t* block_table, void* out, float* lse, void* workspace,
                               size_t workspace_bytes, hipStream_t stream) {
    const int rc = check_plan4(plan);
    if (rc != MSTAR_OK) return rc;
    return mstar::run_fwd(kKernels4, plan, q, k_pages, v_pages, block_table, out, lse, workspace, workspace_bytes,
                          stream, nullptr, nullptr);
}

MSTAR_EXPORT int mstar_kv4_fwd_noalloc(const mstar_plan_t* plan, const void* q, const void* k_pages,
                                       const void* v_pages, const int32_t* block_table, void* out, float* lse,
                                       hipStream_t stream) {
    const int rc = check_plan4(plan);
    if (rc != MSTAR_OK) return rc;
    return mstar::run_fwd_noalloc(kKernels4, plan, q, k_pages, v_pages, block_table, out, lse, stream);
}

MSTAR_EXPORT int mstar_kv4_unpack(int32_t num_kv_heads, int32_t head_dim, int32_t num_pages, const void* k_pages,
                                  const void* v_pages, const int32_t* page_ids, int32_t num_ids, void* k_out,
                                  void* v_out, hipStream_t stream) {
    if (num_kv_heads < 1 || num_pages < 1 || num_ids < 0)
        return fail(MSTAR_ERR_INVALID_ARG, "num_kv_heads and num_pages must be positive, num_ids not negative");
    if (head_dim != 64 && head_dim != 128) return fail(MSTAR_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
    if (num_ids == 0) return MSTAR_OK;
    if (!k_pages || !v_pages || !page_ids || !k_out || !v_out)
        return fail(MSTAR_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(k_out, 16) || !aligned(v_out, 16) ||
        !aligned(page_ids, 4))
        return fail(MSTAR_ERR_INVALID_ARG, "k_pages/v_pages/k_out/v_out must be 16-byte aligned");
    mstar::Unpack4Args a{};
    a.k = k_pages;
    a.v = v_pages;
    a.ids = page_ids;
    a.k_out = k_out;
    a.v_out = v_out;
    a.n_ids = num_ids;
    a.hkv = num_kv_heads;
    a.num_pages = num_pages;
    const hipError_t e = mstar::launch_unpack4(a, head_dim, stream);
    return e == hipSuccess ? MSTAR_OK : hip_fail(e, "4-bit unpack kernel launch");
}

MSTAR_EXPORT int64_t mstar_block_tables_pages(const mstar_plan_t* plan) { return plan ? plan->host.new_pages : 0; }

MSTAR_EXPORT int mstar_block_tables(const mstar_plan_t* plan, const int32_t* free_pages, int64_t num_free,
                                    int32_t* block_table, int64_t* slots, hipStream_t stream) {
    const int rc = check_plan(plan);
    if (rc != MSTAR_OK) return rc;
    const mstar::HostPlan& h = plan->host;
    if (num_free < h.new_pages)
        return fail(MSTAR_ERR_INVALID_ARG, "the step needs " + std::to_string(h.new_pages) + " free pages, " +
                                               std::to_string(num_free) + " are there");
    if (h.appends.empty()) return MSTAR_OK;
    if (!block_table || (h.new_pages > 0 && !free_pages))
        return fail(MSTAR_ERR_INVALID_ARG, "a tensor pointer is NULL");
    if (!aligned(free_pages, 4) || !aligned(block_table, 4) || !aligned(slots, 8))
        return fail(MSTAR_ERR_INVALID_ARG, "free_pages, block_table or slots is misaligned");
    mstar::TablesArgs a{};
    a.seqs = at<const mstar::SeqInfo>(plan, plan->off_seqs);
    a.items = at<const mstar::WorkItem>(plan, plan->off_append);
    a.free_pages = free_pages;
    a.bt = block_table;
    a.slots = slots;
    a.err = at<int32_t>(plan, plan->off_err);
    a.n_items = (int32_t)h.appends.size();
    a.bt_stride = h.params.max_blocks_per_seq;
    a.num_pages = h.params.num_pages;
    hipError_t e = mstar::use_event(plan, stream, &a.done);
    if (e != hipSuccess) return hip_fail(e, "hipStreamIsCapturing");
    if ((e = mstar::launch_tables(a, stream)) != hipSuccess) return hip_fail(e, "block table kernel launch");
    if (a.done) plan->blk->last_use_set = true;
    return MSTAR_OK;
}
