// Device code that the attention kernels share, for gfx950 (CDNA4): 64-lane
// waves, 16x16x32 bf16 MFMA, LDS transpose reads.
//
// Notation used throughout: a 16x16x32 MFMA computes D[16][16] += A[16][32] *
// B[32][16].  Lane l (group G = l / 16, index n = l % 16) supplies
// A[n][8G .. 8G+7] and B[8G .. 8G+7][n], and receives D[4G .. 4G+3][n].
//
// Scores are formed transposed, S^T = K * Q^T (A = 16 keys x 32 dims of K,
// B = 32 dims x 16 query rows of Q^T), so lane l owns query row n and keys
// 4G .. 4G+3 of every 16-key block.  The weighted value sum is likewise
// transposed, O^T = V^T * P^T: the B operand P^T needs exactly the score
// values lane l already holds (two 16-key blocks make one 32-key step), and the
// A operand V^T is read from LDS with ds_read_b64_tr_b16.  Row statistics
// (running max, running sum, rescale factor) are therefore per-lane scalars.
//
// The softmax runs in base 2: s2 = s * sm_scale * log2(e), p = 2^(s2 - m2),
// and lse = (m2 + log2 l) * ln 2 at the end.
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include "kernels.h"

namespace mstar {
namespace {

typedef __bf16 bf16_t;
typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr float kLn2 = 0.6931471805599453f;
constexpr int MSTAR_DEVERR_PAGE_RANGE_BIT = 1;  // MSTAR_DEVERR_PAGE_RANGE
constexpr float kNegInf = -__builtin_inff();

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ f32x4 mfma4(float a, float b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Workgroup and work-item indices straight from the hardware.  The runtime
// library's blockIdx / threadIdx accessors are not inlined into functions built
// with the IEEE mode bit off (their attributes differ), so they would be real
// calls returning the indices in vector registers, and everything derived from
// the workgroup index (item, bounds, loop counts) would leave scalar registers.
__device__ __forceinline__ int wg_id() { return (int)__builtin_amdgcn_workgroup_id_x(); }
__device__ __forceinline__ int thread_id() { return (int)__builtin_amdgcn_workitem_id_x(); }

// Reductions over the four lanes l, l^16, l^32, l^48 that share a query row,
// with gfx950's permlane swaps (v_permlane32_swap exchanges the upper half-wave
// of one register with the lower half of another; with both operands the same
// value, the two results hold x[l] and x[l^32] in some order, and likewise
// for 16).  Sums are formed in the same order on all four lanes.
// IEEE maximumNumber: the hardware max instruction as is.  fmaxf also has to
// quiet signalling NaNs, which costs an extra instruction per operand whenever
// the compiler cannot prove an input is not one (e.g. after a masking select).
__device__ __forceinline__ float fmax_num(float a, float b) { return __builtin_elementwise_maximumnum(a, b); }

struct RowGroup {
    __device__ __forceinline__ static float max(float x) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = fmax_num(__uint_as_float(a[0]), __uint_as_float(a[1]));
        const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return fmax_num(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    __device__ __forceinline__ static float sum(float x) {
        const auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
        const auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        return __uint_as_float(b[0]) + __uint_as_float(b[1]);
    }
};

__device__ __forceinline__ bf16x4 lds_read_tr16(const bf16_t* p) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p));
}

__device__ __forceinline__ bf16x8 cat(bf16x4 a, bf16x4 b) {
    return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}

__device__ __forceinline__ bf16x8 to_bf16x8(f32x4 a, f32x4 b) {
    return cat(__builtin_convertvector(a, bf16x4), __builtin_convertvector(b, bf16x4));
}

// K/V rows are read through a buffer resource per page: the page base lives in
// scalar registers (built with scalar ops from the wave-uniform page index) and
// each lane adds a 32-bit byte offset that does not change from tile to tile,
// so the loads cost no vector ALU work.  The resource's range is one page.
constexpr int kBufferDword3 = 0x00020000;  // gfx9 buffer resource word 3 (raw, no format)

__device__ __forceinline__ __amdgpu_buffer_rsrc_t page_rsrc(const char* base, size_t byte_ofs, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base + byte_ofs), (short)0, (int)bytes,
                                             kBufferDword3);
}

__device__ __forceinline__ uint4 load16_at(__amdgpu_buffer_rsrc_t r, uint32_t byte_off) {
    return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, (int)byte_off, 0, 0));
}

__device__ __forceinline__ uint4 load16(const void* base, int64_t elem_off_bf16) {
    return *reinterpret_cast<const uint4*>(reinterpret_cast<const bf16_t*>(base) + elem_off_bf16);
}
// The same with the non-temporal hint: for data read once (a tile's Q rows),
// so that it does not push shared K/V lines out of the caches (text+latent
// launch: fetched bytes 527 -> 334 MB, of which 250 MB are Q).
__device__ __forceinline__ uint4 load16_nt(const void* base, int64_t elem_off_bf16) {
    typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
    const u32x4 w =
        __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(reinterpret_cast<const bf16_t*>(base) + elem_off_bf16));
    return __builtin_bit_cast(uint4, w);
}

// Visible interval of query row i of a request, clipped to the item's keys.
__device__ __forceinline__ void row_interval(const KArgs& a, const SeqInfo& si, const WorkItem& it,
                                             int32_t i, int32_t& lo, int32_t& hi) {
    const int32_t pos = si.kv_len - si.q_len + i;
    int32_t l0 = si.window > 0 ? max(0, pos - si.window + 1) : 0;
    int32_t h0 = a.row_hi[si.hi_off + i];
    lo = max(l0, it.k_begin);
    hi = min(h0, it.k_end);
}

// p / group of a (query row, head) pair index p of an item: a multiply by the
// host's reciprocal, exact below 2^32 / group.
__device__ __forceinline__ int div_group(const KArgs& a, int p) {
    if (a.group_inv == 0) return a.group == 1 ? p : p / a.group;
    return (int)(((uint64_t)(uint32_t)p * a.group_inv) >> 32);
}

// Lazy reference threshold (base-2 units): the online softmax moves its
// reference max only when a row's max exceeds it by more than this, so
// probabilities taken against a stale reference stay below 2^kLazy.
constexpr float kLazy = 8.0f;

// Balanced reductions over the 4*NB score values a lane holds for one row.
// Three-input maximum (one v_max3_f32).
__device__ __forceinline__ float max3(float a, float b, float c) { return fmax_num(fmax_num(a, b), c); }
template <int NB>
__device__ __forceinline__ float tree_max(const f32x4 (&s)[NB]) {
    static_assert(NB == 2 || NB == 4, "tree shapes for 8 and 16 values");
    if constexpr (NB == 4) {  // 16 values: 5 + 2 three-input maxima and one pair
        const float a0 = max3(s[0][0], s[0][1], s[0][2]), a1 = max3(s[0][3], s[1][0], s[1][1]);
        const float a2 = max3(s[1][2], s[1][3], s[2][0]), a3 = max3(s[2][1], s[2][2], s[2][3]);
        const float a4 = max3(s[3][0], s[3][1], s[3][2]);
        return fmax_num(max3(a0, a1, a2), max3(a3, a4, s[3][3]));
    } else {  // 8 values: two three-input maxima and one more over the rest
        const float a0 = max3(s[0][0], s[0][1], s[0][2]), a1 = max3(s[0][3], s[1][0], s[1][1]);
        return max3(a0, a1, fmax_num(s[1][2], s[1][3]));
    }
}
template <int NB>
__device__ __forceinline__ float tree_sum(const f32x4 (&s)[NB]) {
    float v[NB];
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) v[kb] = (s[kb][0] + s[kb][1]) + (s[kb][2] + s[kb][3]);
#pragma unroll
    for (int w = NB / 2; w >= 1; w /= 2)
#pragma unroll
        for (int kb = 0; kb < w; ++kb) v[kb] = v[kb] + v[kb + w];
    return v[0];
}

// Online-softmax update of all RB 16-row blocks a wave owns, each with NB
// 16-key blocks of raw scores (hidden keys already -inf).  m and l are kept
// in base-2 units of the scaled scores: c = sm_scale * log2(e) > 0, so
// max(c s) = c max(s) and every probability is one FMA and one exp2.  The row
// blocks are processed side by side and reductions are balanced trees, so the
// dependency chains stay short.
//
// The reference max m is refreshed lazily: only when some row of the wave
// sees its max grow by more than kLazy (or has no reference yet).  Otherwise
// probabilities are taken against the stale m, so they stay below 2^kLazy, and
// the rescale of the O accumulators (the most expensive VALU work per tile)
// is skipped.  The result is exact either way: out = O / l and
// lse = m + log2(l) use the same reference.  Returns true (wave-uniform) when
// every O block rb must be multiplied by alpha[rb].  Leaves the probabilities
// in s.
template <int RB, int NB>
__device__ __forceinline__ bool softmax_update(const RowGroup& rg, f32x4 (&s)[RB][NB], float c, float (&m)[RB],
                                               float (&l)[RB], float (&alpha)[RB]) {
    float mx[RB];
    bool grow = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) mx[rb] = tree_max<NB>(s[rb]);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        mx[rb] = rg.max(mx[rb]) * c;
        grow |= mx[rb] > m[rb] + kLazy;  // false while both are -inf
    }
    const bool rescale = __builtin_amdgcn_ballot_w64(grow) != 0;
    float m_use[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        alpha[rb] = 1.0f;
        if (rescale) {
            const float m_new = fmax_num(m[rb], mx[rb]);
            alpha[rb] = fast_exp2(m[rb] - (m_new == kNegInf ? 0.0f : m_new));
            m[rb] = m_new;
        }
        m_use[rb] = m[rb] == kNegInf ? 0.0f : m[rb];
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[rb][kb][i] = fast_exp2(fmaf(s[rb][kb][i], c, -m_use[rb]));
    // The sums are taken over the fp32 probabilities, not over their bf16
    // roundings that enter P.V: a row dominated by a few keys would otherwise
    // carry up to 2^-9 relative error into lse.
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float sum = tree_sum<NB>(s[rb]);  // per-lane partial; row total reduced at the end
        l[rb] = rescale ? l[rb] * alpha[rb] + sum : l[rb] + sum;
    }
    return rescale;
}

// Probabilities against a fixed per-row reference m: p = 2^(c s - m), with no
// maximum; hidden keys are -inf and give 0.  ts receives the lane's partial
// sums of the tile.
template <int RB, int NB>
__device__ __forceinline__ void softmax_fixed(f32x4 (&s)[RB][NB], float c, const float (&m)[RB], float (&ts)[RB]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int kb = 0; kb < NB; ++kb)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[rb][kb][i] = fast_exp2(fmaf(s[rb][kb][i], c, -m[rb]));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) ts[rb] = tree_sum<NB>(s[rb]);
}
// Bound on a lane's partial sum of one tile under the fixed reference: below
// it every probability is below 2^32, far from overflow of the sums and the
// weighted values; at or above it (or inf / NaN) the tile is redone exactly.  A
// row's weights then sum to less than 2^60 over any 2^31 keys (2^26 tiles of 32, four
// lanes each), so that weighted sums of values up to 2^64 stay below 2^124: the
// range that a 4-bit cache states, whose format reaches 6 * 2^125 (values of
// 2^100 under scores that grow by a few units gave infinities).
constexpr float kFixedTileLimit = 4294967296.0f;  // 2^32

template <int D>
__device__ __forceinline__ int k_swizzle(int row) {  // 16-byte chunk XOR for K rows
    return D == 128 ? (row & 15) : ((row >> 1) & 7);
}
template <int D>
__device__ __forceinline__ int v_swizzle(int row) {  // 16-byte chunk XOR for V rows (even: 32-byte pairs stay whole)
    return D == 128 ? ((row & 7) << 1) : (((row >> 1) & 3) << 1);
}

// 4-byte direct global -> LDS load of one wave: lane i writes LDS bytes
// [lds_addr + 4 i, +4).  Issued from assembly so that the compiler does not
// track it (a tracked load in the tile loop makes the compiler wait for every
// outstanding load before its result is first used); the kernel waits itself
// (dma_barrier) before reading the filled bytes.
__device__ __forceinline__ void lds_dma4(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t lds_addr) {
    // M0 holds the (wave-uniform) LDS address; the compiler reserves M0, so
    // the asm puts its previous value back instead of declaring it clobbered
    uint32_t saved;
    asm volatile(
        "s_mov_b32 %0, m0\n\t"
        "s_mov_b32 m0, %3\n\t"
        "buffer_load_dword %1, %2, 0 offen lds\n\t"
        "s_mov_b32 m0, %0"
        : "=&s"(saved)
        : "v"(voff), "s"(r), "s"(__builtin_amdgcn_readfirstlane(lds_addr))
        : "memory");
}
// Waits for this wave's direct loads and LDS reads, then for the workgroup.
__device__ __forceinline__ void dma_barrier() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
// The same without the wait for loads: for tiles that waves write into LDS themselves.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }
typedef __attribute__((address_space(3))) char lds_char;

// Waits until at most N vector memory operations of this wave are outstanding.
template <int N>
__device__ __forceinline__ void wait_vmem() {
    static_assert(N >= 0 && N < 16, "vmcnt immediate");
    // gfx9 s_waitcnt encoding: vmcnt[3:0] in bits 3:0, expcnt and lgkmcnt at
    // their no-wait maxima (7 in bits 6:4, 15 in bits 11:8)
    __builtin_amdgcn_s_waitcnt(N | (7 << 4) | (15 << 8));
}

// 16-byte direct global -> LDS load of one wave through the compiler's
// builtin (lane i writes bytes [16 i, 16 i + 16) after `lds`, which must be
// wave-uniform).  The compiler tracks it and waits for it before later LDS
// reads.  The load is marked non-temporal (the NT cache-policy bit): the few-row
// kernel reads each V row of a request once, so its lines go first when the
// caches need room (decode batch: 0.617 -> 0.676 of HBM peak; 16-token
// chunks: 0.593 -> 0.618).  Marking the K loads into registers as well was
// slower on the chunk batch (0.571).
constexpr int kCachePolicyNT = 2;
__device__ __forceinline__ void lds_load16_nt(__amdgpu_buffer_rsrc_t r, uint32_t voff, void* lds) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(lds), 16, voff, 0, 0,
                                             kCachePolicyNT);
}
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const lds_char*)(p);
}
// 16-byte direct load with a wave-uniform scalar byte offset added to the
// global address, issued from assembly with the LDS address in M0.  The
// compiler waits for a direct load it tracks before any later LDS read that
// it cannot prove disjoint, and without alias-scope information it proves
// none: through the builtin, the next tile's prefetch made every tile wait
// for that prefetch before its first K read (text+latent 1.790 -> 1.709 ms
// together with the page indices read a tile ahead).  This one is not
// tracked; the caller waits itself (dma_barrier) before anything reads the
// bytes it writes.
__device__ __forceinline__ void lds_dma16s(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff, uint32_t lds_addr) {
    asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds"
                 :
                 : "v"(voff), "s"(r), "s"(soff), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr))
                 : "memory");
}

// K/V of a pool that fits in 2 GB are read through one buffer resource per
// pool with the page's byte offset in the instruction's scalar offset, so a
// load costs no scalar work beyond one multiply per page.  Larger pools get a
// resource per page.  The 2 GB resource range keeps every
// valid offset in range and pushes the marker offset below out of range.
constexpr uint32_t kSmallPoolBytes = 0x80000000u;

// Launches `kernel`; the event a.done, if given, completes with it.  It rides on
// the dispatch itself: recorded behind it, it would be a packet of its own that
// keeps the next kernel waiting (2.9 us a call; each kv_append and fwd marks its
// plan's use this way).  Not for streams under capture.
template <typename Args>
hipError_t launch(void (*kernel)(Args), dim3 grid, dim3 block, const Args& a, hipStream_t s) {
    void* args[] = {const_cast<Args*>(&a)};
    const void* fn = reinterpret_cast<const void*>(kernel);
    return a.done ? hipExtLaunchKernel(fn, grid, block, args, 0, s, nullptr, a.done, 0)
                  : hipLaunchKernel(fn, grid, block, args, 0, s);
}

}  // namespace
}  // namespace mstar
