// HIP kernels for batched paged attention with per-row visible intervals,
// written for gfx950 (CDNA4); the multi-row tile kernel is in tile.h.

#include <mutex>

#include "kernels.h"
#include "tile.h"

// Device scratch of the allocation-free entry point: the split-K partials of
// one call (fp32 partial rows, then their log-sum-exps) live here instead of
// in a caller workspace.  One copy per GPU, held until the process ends.  In
// host code this name is a host-side stand-in, never a device address: the
// device address comes from hipGetSymbolAddress (scratch_buffer below).
static __device__ __align__(256) unsigned char scratch[mstar::kScratchBytes];

namespace mstar {
namespace {

// ---------------------------------------------------------------------------
// Few-row kernel: one workgroup = up to 16*RB rows (query rows x the query
// heads of one KV head) against the item's key range.  The four waves take
// interleaved 32-key steps; K goes straight from HBM into MFMA operand
// registers, V straight into a wave-private LDS slot for the transpose read.
// The four waves' partial results are combined through LDS.
//
// Bound: HBM.  One step is in flight per wave: its registers and its V slot take
// the next step's loads as soon as they are read.  A second set of both bought
// nothing, since a wave waits for all of its loads before each step (see
// compute_step), and cost a workgroup per CU and the room beside the tile
// kernel: 48 decode steps and 64 chunks beside one image and 16 rollouts in
// one launch 622 -> 574 us, 16 decode steps at D = 64 28.7 -> 27.3, a decode
// batch of 64 120.5 -> 121.1 (5.1 TB/s either way).
// ---------------------------------------------------------------------------
template <int D, int RB>
__global__ __launch_bounds__(256, RB == 1 ? 3 : 2) void few_kernel(KArgs a) {
    constexpr int NW = 4;             // waves
    constexpr int SK = kSubKeys;
    constexpr int RBY = 2 * D;        // bytes per V row in LDS
    constexpr int DS = D / 32, DB = D / 16, CH = D / 8;
    constexpr int VL = SK * CH / 64;  // direct V loads per wave and step
    constexpr int RPL = 64 / CH;      // V rows filled by one wave-wide load
    // Bytes of one wave's V slot, 5/16 more than it holds: that keeps D =
    // 128 at three workgroups per CU, which share out a batch cut
    // into 768 pieces better than four do (decode batch of 64: 121 us, against
    // 129 with four and 512 or 127 with four and 768 pieces; four need 1536
    // pieces and their merge for the same 121).
    constexpr int SB = SK * RBY * 21 / 16;
    static_assert(16 * D * 4 <= SB, "a wave's V slot takes 16 rows of its results");
    static_assert(SB % 256 == 0, "V slots start on a row of LDS banks");
    __shared__ __attribute__((aligned(1024))) char v_slot[NW][SB];
    __shared__ float ml_lds[NW][2][RB * 16];
    __shared__ float fin_lds[2][RB * 16];

    const WorkItem it = a.items[wg_id()];
    const SeqInfo si = a.seqs[it.seq];
    const int tid = thread_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6) & (NW - 1), lane = tid & 63;
    const int n = lane & 15, grp = lane >> 4;
    const int G = a.group;
    const int kvh = it.head;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    const RowGroup rg;

    int32_t lo[RB], hi[RB];
    bool valid[RB];
    bf16x8 qf[RB][DS];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = rb * 16 + n;
        valid[rb] = r < it.nrows;
        const int rr = it.row0 + r;
        const int qi = rr / G, h = kvh * G + rr % G;
        lo[rb] = 0;
        hi[rb] = 0;
        if (valid[rb]) row_interval(a, si, it, qi, lo[rb], hi[rb]);
        const int64_t qoff = ((int64_t)(si.q_start + qi) * a.hq + h) * D;
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            if (valid[rb]) {
                qf[rb][s] = __builtin_bit_cast(bf16x8, load16(a.q, qoff + 32 * s + 8 * grp));
            } else {
                qf[rb][s] = bf16x8{};
            }
        }
    }
    int32_t lo_max, hi_min, dummy;
    {
        const int q_first = it.row0 / G, q_last = (it.row0 + it.nrows - 1) / G;
        row_interval(a, si, it, q_first, dummy, hi_min);
        row_interval(a, si, it, q_last, lo_max, dummy);
    }

    float m[RB], l[RB];
    f32x4 o[RB][DB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = kNegInf;
        l[rb] = 0.0f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0, 0, 0, 0};
    }

    // Wave w takes steps w, w + NW, w + 2 NW, ... of 32 keys; its i-th step starts
    // at key k_begin + 32 * (w + NW i) and spans exactly two pages (k_begin is page
    // aligned).  The page indices of 32 consecutive steps live in one register
    // (lane 2i+h holds half h of step i) and are read back with readlane, so no
    // block-table load sits between a step and its K/V loads.
    const int n_steps = (it.k_end - it.k_begin + SK - 1) / SK;
    const int my_steps = wave < n_steps ? (n_steps - wave + NW - 1) / NW : 0;
    const int32_t page0 = it.k_begin >> 4;
    const int32_t n_pages = ((it.k_end + 15) >> 4) - page0;
    auto load_pages = [&](int first_step) {
        const int pg = 2 * (wave + NW * (first_step + (lane >> 1))) + (lane & 1);
        return pg < n_pages ? bt_row[page0 + pg] : 0;
    };
    int32_t pw_cur = load_pages(0), pw_next = my_steps > 32 ? load_pages(32) : 0;
    const int64_t slot_stride = (int64_t)a.hkv * D;

    // K of one step, straight into MFMA operand registers
    struct Step {
        uint4 k[2][DS];
    };
    // Byte offsets of this lane's K and V chunks inside their page, the same
    // for every step; the page (wave-uniform) supplies a scalar base.  Rows past
    // the item's end read zeros through the buffer range check and a page
    // outside the pool gets an empty range, so the data needs no selects.
    constexpr uint32_t kOutOfRange = 0x80000000u;
    const size_t page_bytes = (size_t)16 * slot_stride * sizeof(bf16_t);
    uint32_t koff[DS];
#pragma unroll
    for (int s = 0; s < DS; ++s)
        koff[s] = (uint32_t)((n * slot_stride + (int64_t)kvh * D + 32 * s + 8 * grp) * sizeof(bf16_t));
    // V load j fills rows j RPL .. j RPL + RPL - 1 of the step; the lane writes
    // physical chunk lane % CH of its row and fetches the logical chunk that the
    // row's swizzle puts there.  The in-page slot and the swizzle repeat every
    // 16 / RPL loads.
    constexpr int VJ = 16 / RPL;
    uint32_t voff[VJ];
#pragma unroll
    for (int j = 0; j < VJ; ++j) {
        const int row = j * RPL + lane / CH;
        const int chunk = (lane % CH) ^ v_swizzle<D>(row);
        voff[j] = (uint32_t)(((row & 15) * slot_stride + (int64_t)kvh * D + 8 * chunk) * sizeof(bf16_t));
    }
    // transposing V reads: rows 4 grp + n / 4 (+16), bf16 columns 16 db + 4 (n & 3)
    uint32_t vrd[DB];
    {
        const int vr = 4 * grp + (n >> 2);
        const int vh = v_swizzle<D>(vr) >> 1;
        const uint32_t base = vr * RBY + (((n & 3) >> 1) << 4) + ((n & 1) << 3);
#pragma unroll
        for (int db = 0; db < DB; ++db) vrd[db] = base + ((db ^ vh) << 5);
    }
    const int wave_u = __builtin_amdgcn_readfirstlane(wave);
    const char* kbase = reinterpret_cast<const char*>(a.k);
    const char* vbase = reinterpret_cast<const char*>(a.v);
    bool page_err = false;
    Step st;
    __amdgpu_buffer_rsrc_t rv[2];
    auto load_k = [&](int i) {  // also the step's V pages, for load_v
        if (i > 0 && (i & 31) == 0) {  // next window of page indices
            pw_cur = pw_next;
            pw_next = i + 32 < my_steps ? load_pages(i + 32) : 0;
        }
        const int32_t k0 = it.k_begin + SK * (wave + NW * i);
        const bool tail = k0 + SK > it.k_end;
        __amdgpu_buffer_rsrc_t rk[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int32_t page = __builtin_amdgcn_readlane(pw_cur, 2 * (i & 31) + h);
            const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
            page_err |= !ok && k0 + 16 * h < it.k_end;
            const size_t pofs = ok ? (size_t)page * page_bytes : 0;
            const uint32_t nrec = ok ? (uint32_t)page_bytes : 0u;
            rk[h] = page_rsrc(kbase, pofs, nrec);
            rv[h] = page_rsrc(vbase, pofs, nrec);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const bool live = !tail || k0 + kb * 16 + n < it.k_end;
#pragma unroll
            for (int s = 0; s < DS; ++s) st.k[kb][s] = load16_at(rk[kb], live ? koff[s] : kOutOfRange);
        }
    };
    auto load_v = [&](int i) {
        const int32_t k0 = it.k_begin + SK * (wave + NW * i);
        const bool tail = k0 + SK > it.k_end;
#pragma unroll
        for (int j = 0; j < VL; ++j) {
            const int row = j * RPL + lane / CH;
            const int h = (j * RPL) >> 4;  // page half of the load's rows: the same across the wave
            const bool live = !tail || k0 + row < it.k_end;
            lds_load16_nt(rv[h], live ? voff[j % VJ] : kOutOfRange, &v_slot[wave_u][j * 1024]);
        }
    };

    auto compute_step = [&](int i) {
        // Wait for every outstanding load of this wave, K registers and V
        // slot alike, before the step.  A partial wait that counts other
        // loads as younger (what the compiler emits, and tighter forms
        // of it) has produced stale V on this hardware when direct-to-LDS
        // loads and loads into registers are in flight together, so the
        // kernel does not rely on their relative completion order.
        wait_vmem<0>();
        const int32_t k0 = it.k_begin + SK * (wave + NW * i);
        f32x4 sc[RB][2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const bf16x8 kf = __builtin_bit_cast(bf16x8, st.k[kb][s]);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
                    sc[rb][kb] = mfma16(kf, qf[rb][s], s == 0 ? f32x4{0, 0, 0, 0} : sc[rb][kb]);
            }
        if (i + 1 < my_steps) load_k(i + 1);  // the K registers are free

        const bool full = k0 >= lo_max && k0 + SK <= hi_min;
        if (!full) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int32_t lo_r = lo[rb] - (k0 + 4 * grp), hi_r = hi[rb] - (k0 + 4 * grp);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = kb * 16 + e;
                        if (!(c >= lo_r && c < hi_r)) sc[rb][kb][e] = kNegInf;
                    }
            }
        }
        float alpha[RB];
        if (softmax_update<RB, 2>(rg, sc, a.scale_log2, m, l, alpha)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int db = 0; db < DB; ++db) o[rb][db] *= alpha[rb];
        }
        bf16x8 pf[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) pf[rb] = to_bf16x8(sc[rb][0], sc[rb][1]);
#pragma unroll
        for (int db = 0; db < DB; ++db) {
            const bf16_t* base = reinterpret_cast<const bf16_t*>(&v_slot[wave][vrd[db]]);
            const bf16x8 vf = cat(lds_read_tr16(base), lds_read_tr16(base + 16 * D));
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) o[rb][db] = mfma16(vf, pf[rb], o[rb][db]);
        }
        // the V slot is free once this wave's reads of it have returned
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (i + 1 < my_steps) load_v(i + 1);
    };

    if (my_steps > 0) {
        load_k(0);
        load_v(0);
    }
    for (int i = 0; i < my_steps; ++i) compute_step(i);

    if (page_err && lane == 0) atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);

    // ---- combine the waves -------------------------------------------------------
    float lt[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) lt[rb] = rg.sum(l[rb]);
    if (grp == 0) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            ml_lds[wave][0][rb * 16 + n] = m[rb];
            ml_lds[wave][1][rb * 16 + n] = lt[rb];
        }
    }
    __syncthreads();
    // one row block at a time: each wave leaves its results, against the common
    // reference, in its own V slot (16-byte pieces in lane order: no bank
    // conflicts), and all threads add the waves' pieces up.  (One wave after the
    // other into row-major sums took 1-2 us more per workgroup: 16 16-token
    // chunks 40 -> 35 us, a decode batch of 64 121.2 -> 120.2.)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = rb * 16 + n;
        float mstar = kNegInf;
#pragma unroll
        for (int w = 0; w < NW; ++w) mstar = fmax_num(mstar, ml_lds[w][0][row]);
        const float mu = mstar == kNegInf ? 0.0f : mstar;
        if (wave == 0 && grp == 0) {
            float L = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) L += fast_exp2(ml_lds[w][0][row] - mu) * ml_lds[w][1][row];
            fin_lds[0][row] = mstar;
            fin_lds[1][row] = L;
        }
        const float own = fast_exp2(m[rb] - mu);
        f32x4* slot = reinterpret_cast<f32x4*>(&v_slot[wave][0]);
        if (rb > 0) __syncthreads();  // the previous block has been added up
#pragma unroll
        for (int db = 0; db < DB; ++db) slot[db * 64 + lane] = o[rb][db] * own;
        __syncthreads();
        for (int e = tid; e < DB * 64; e += 64 * NW) {
            const int r = rb * 16 + (e & 15), d4 = (e >> 6) * 16 + 4 * ((e >> 4) & 3);
            if (r >= it.nrows) continue;
            f32x4 val = reinterpret_cast<const f32x4*>(&v_slot[0][0])[e];
#pragma unroll
            for (int w = 1; w < NW; ++w) val += reinterpret_cast<const f32x4*>(&v_slot[w][0])[e];
            const float L = fin_lds[1][r];
            val *= L > 0.0f ? 1.0f / L : 0.0f;
            const float lse = L > 0.0f ? (fin_lds[0][r] + __log2f(L)) * kLn2 : kNegInf;
            const int rr = it.row0 + r;
            if (it.part < 0) {
                const int64_t orow = (int64_t)(si.q_start + rr / G) * a.hq + kvh * G + rr % G;
                *reinterpret_cast<bf16x4*>(reinterpret_cast<bf16_t*>(a.out) + orow * D + d4) =
                    __builtin_convertvector(val, bf16x4);
                if (d4 == 0) a.lse[orow] = lse;
            } else {
                const int64_t slot_r = it.part + r;
                *reinterpret_cast<f32x4*>(a.part_o + slot_r * D + d4) = val;
                if (d4 == 0) a.part_lse[slot_r] = lse;
            }
        }
    }
}

// ---------------------------------------------------------------------------
// fp32 kernel: one workgroup = up to 16 (query row, head) rows of one KV head
// against every key they see; its waves take interleaved 16-key steps (one
// page each) and their results are combined through LDS.
//
// Both products run on 16x16x4 fp32 MFMAs, which multiply and accumulate in
// full fp32: lane l (group G = l / 16, n = l % 16) supplies A[n][G] and
// B[G][n] and receives D[4G .. 4G+3][n].  The order of a contraction is free,
// so both operands of a step come from 16-byte loads: scores S^T = K Q^T take
// dims 16 j + 4 G + c in step (j, c) (lane n reads its key's 16 bytes at dim
// 16 j + 4 G); values O^T = V^T P^T take key 4 G + c in step c, whose
// probability the lane already holds, and output row m of block (h, e) stands
// for dim 64 h + 4 m + e (lane n reads key 4 G + c's 16 bytes at dim 64 h +
// 4 n).  K and V go straight into registers; nothing passes through LDS but
// the combine.
//
// Bound: latency inside a step, not a rate.  Four prompts of 246-782 tokens and
// four decode rows (8/2 heads, D = 128: 2.3 GFLOP) keep the matrix units busy a
// third of the time (64 MFMAs of 32 cycles per 16 rows x 16 keys; the CU with
// the most has 21 us of them) and read 10-13 bytes per clock and CU from L2, of
// about 64; waves spend 0.40 of their time waiting for loads and barriers and
// 0.47 for an issue slot.  One wave per (row, head) with scalar dot products,
// each reading all of its keys by itself, took 350 us for it where this takes
// 41; four prompts of 5-64 tokens at D = 64: 8.1 -> 5.5 us.  Four waves per
// workgroup: eight have the longest item done sooner, but only one such
// workgroup fits a CU at D = 128, which bares every item's first loads and its
// combine (55 us).
// ---------------------------------------------------------------------------
template <int D, int NW>
__global__ __launch_bounds__(64 * NW, D == 64 ? 4 : 3) void f32_kernel(KArgs a) {
    constexpr int KJ = D / 16;  // 16-byte K (and Q) pieces per lane
    constexpr int VH = D / 64;  // 16-byte V pieces per lane and key
    __shared__ __attribute__((aligned(16))) float o_lds[NW][16 * D];
    __shared__ float ml_lds[2][NW][16];

    const WorkItem it = a.items[wg_id()];
    const SeqInfo si = a.seqs[it.seq];
    // The item stands for query rows row0 .. row0 + nrows - 1 of one head; the
    // G items of a KV head's group share their (row, head) pairs out as slices
    // of 16, so that one read of K and V serves rows of several heads.  Items
    // past the last slice have nothing to do.
    const int G = a.group;
    const int kvh = it.head / G;
    const int p0 = (it.head - kvh * G) * 16;
    const int np = min(it.nrows * G - p0, 16);
    if (np <= 0) return;
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & (NW - 1), lane = thread_id() & 63;
    const int n = lane & 15, grp = lane >> 4;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    const RowGroup rg;

    // ---- this lane's row; the slice's bounds (intervals never shrink) ---------
    const bool valid = n < np;
    const int pr = p0 + (valid ? n : 0);
    const int pq = div_group(a, pr), qi = it.row0 + pq, head = kvh * G + pr - pq * G;
    int32_t lo, hi, lo_min, lo_max, hi_min, hi_max;
    row_interval(a, si, it, qi, lo, hi);
    if (!valid) lo = hi = 0;
    row_interval(a, si, it, it.row0 + div_group(a, p0), lo_min, hi_min);
    row_interval(a, si, it, it.row0 + div_group(a, p0 + np - 1), lo_max, hi_max);
    float4 qf[KJ];
    {
        const float* q = reinterpret_cast<const float*>(a.q) + ((int64_t)(si.q_start + qi) * a.hq + head) * D;
#pragma unroll
        for (int j = 0; j < KJ; ++j)
            qf[j] = valid ? *reinterpret_cast<const float4*>(q + 16 * j + 4 * grp) : float4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    const int32_t k_first = __builtin_amdgcn_readfirstlane(lo_min & ~(kPage - 1));
    const int32_t k_last = __builtin_amdgcn_readfirstlane(hi_max);
    lo_max = __builtin_amdgcn_readfirstlane(lo_max);
    hi_min = __builtin_amdgcn_readfirstlane(hi_min);

    // ---- steps of this wave: page wave + NW i of the slice's pages ------------
    const int n_pages = (k_last - k_first + kPage - 1) / kPage;
    const int my_steps = wave < n_pages ? (n_pages - wave + NW - 1) / NW : 0;
    const int32_t* bt_first = bt_row + (k_first >> 4);
    auto load_pages = [&](int first) {  // lane i: the page of step first + i
        const int pg = wave + NW * (first + lane);
        return pg < n_pages ? bt_first[pg] : 0;
    };
    int32_t pw = load_pages(0);
    constexpr uint32_t kOutOfRange = 0x80000000u;
    const size_t page_bytes = (size_t)kPage * a.hkv * D * sizeof(float);
    const uint32_t row_bytes = (uint32_t)(a.hkv * D * sizeof(float));
    const uint32_t koff = n * row_bytes + (uint32_t)(kvh * D + 4 * grp) * 4u;
    const uint32_t voff = 4 * grp * row_bytes + (uint32_t)(kvh * D + 4 * n) * 4u;
    const char* kbase = reinterpret_cast<const char*>(a.k);
    const char* vbase = reinterpret_cast<const char*>(a.v);
    bool page_err = false;
    uint4 kr[KJ], vr[4][VH];  // K and V of one step
    // Rows past the slice's last key and pages outside the pool read as zeros
    // through the buffer range check.
    auto step_page = [&](int i, uint32_t& nrec) -> size_t {
        const int32_t page = __builtin_amdgcn_readlane(pw, i & 63);
        const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
        page_err |= !ok;
        nrec = ok ? (uint32_t)page_bytes : 0u;
        return ok ? (size_t)page * page_bytes : 0;
    };
    auto load_k = [&](int i) {
        if (i > 0 && (i & 63) == 0) pw = load_pages(i);
        uint32_t nrec;
        const size_t pofs = step_page(i, nrec);
        const __amdgpu_buffer_rsrc_t rk = page_rsrc(kbase, pofs, nrec);
        const int32_t left = k_last - (k_first + kPage * (wave + NW * i));  // live keys of the step, if below 16
        const uint32_t ko = n < left ? koff : kOutOfRange;
#pragma unroll
        for (int j = 0; j < KJ; ++j) kr[j] = load16_at(rk, ko + 64 * j);
    };
    auto load_v = [&](int i) {  // after load_k(i): the page window holds step i
        uint32_t nrec;
        const size_t pofs = step_page(i, nrec);
        const __amdgpu_buffer_rsrc_t rv = page_rsrc(vbase, pofs, nrec);
        const int32_t left = k_last - (k_first + kPage * (wave + NW * i));
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t vo = 4 * grp + c < left ? voff + c * row_bytes : kOutOfRange;
#pragma unroll
            for (int h = 0; h < VH; ++h) vr[c][h] = load16_at(rv, vo + 256 * h);
        }
    };

    float m = kNegInf, l = 0.0f;
    f32x4 o[VH][4];
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[h][e] = f32x4{0, 0, 0, 0};
    // scores of step i against this lane's row, hidden keys -inf; returns whether no key of the step is hidden
    auto scores = [&](int i, f32x4& s) {
        const int32_t k0 = k_first + kPage * (wave + NW * i);
        f32x4 sa = {0, 0, 0, 0}, sb = {0, 0, 0, 0};  // two chains
#pragma unroll
        for (int j = 0; j < KJ; j += 2) {
            const float4 ka = __builtin_bit_cast(float4, kr[j]), kb = __builtin_bit_cast(float4, kr[j + 1]);
            sa = mfma4(ka.x, qf[j].x, sa);
            sb = mfma4(kb.x, qf[j + 1].x, sb);
            sa = mfma4(ka.y, qf[j].y, sa);
            sb = mfma4(kb.y, qf[j + 1].y, sb);
            sa = mfma4(ka.z, qf[j].z, sa);
            sb = mfma4(kb.z, qf[j + 1].z, sb);
            sa = mfma4(ka.w, qf[j].w, sa);
            sb = mfma4(kb.w, qf[j + 1].w, sb);
        }
        s = sa + sb;
        const bool full = k0 >= lo_max && k0 + kPage <= hi_min;
        if (!full) {
            const int32_t lo_r = lo - (k0 + 4 * grp), hi_r = hi - (k0 + 4 * grp);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (!(c >= lo_r && c < hi_r)) s[c] = kNegInf;
        }
        return full;
    };
    // Probabilities against this lane's reference m, the largest unscaled score
    // so far.  The difference is taken before it is scaled: a scaled score is
    // off by half an ulp, 2^(e - 24) for one near 2^e, and against a reference
    // rounded on its own that alone takes 2^x past the largest float from
    // scores of 2^31 on.  Hidden keys stay at -inf.
    auto probs = [&](const f32x4& s) {
        const float mu = m == kNegInf ? 0.0f : m;
        f32x4 p;
#pragma unroll
        for (int c = 0; c < 4; ++c) p[c] = fast_exp2((s[c] - mu) * a.scale_log2);
        return p;
    };
    bool by_key = false;  // wave-uniform: a value that is not finite in a step with hidden keys
    // Steps: V is requested before the scores, which cover its latency, the
    // next step's K before the weighted values, which cover that one: one
    // register copy of each, so that three waves fit a SIMD at D = 128.
    if (my_steps > 0) load_k(0);
    for (int i = 0; i < my_steps; ++i) {
        load_v(i);
        f32x4 s;
        const bool full = scores(i, s);
        if (i + 1 < my_steps) load_k(i + 1);
        if (!full) {
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int h = 0; h < VH; ++h) {
                    const uint4 w = vr[c][h];
                    top = max(max(top, max(w.x & 0x7fffffffu, w.y & 0x7fffffffu)),
                              max(w.z & 0x7fffffffu, w.w & 0x7fffffffu));
                }
            by_key |= __builtin_amdgcn_ballot_w64(top >= 0x7f800000u) != 0;
        }
        // The reference follows every growth (no lazy threshold): probabilities
        // stay at or below 1, so values as large as the type holds do not
        // overflow, and the rescale is small beside a step's products.
        const float mx = rg.max(fmax_num(fmax_num(s[0], s[1]), fmax_num(s[2], s[3])));
        if (__builtin_amdgcn_ballot_w64(mx > m) != 0) {
            const float m_new = fmax_num(m, mx);
            const float alpha = fast_exp2((m - (m_new == kNegInf ? 0.0f : m_new)) * a.scale_log2);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int h = 0; h < VH; ++h)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[h][e] *= alpha;
        }
        const f32x4 p = probs(s);
        l += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int h = 0; h < VH; ++h) {
                const float4 vv = __builtin_bit_cast(float4, vr[c][h]);
                o[h][0] = mfma4(vv.x, p[c], o[h][0]);
                o[h][1] = mfma4(vv.y, p[c], o[h][1]);
                o[h][2] = mfma4(vv.z, p[c], o[h][2]);
                o[h][3] = mfma4(vv.w, p[c], o[h][3]);
            }
    }
    if (__builtin_expect(by_key, 0)) {
        // An infinite or NaN value must not reach the rows its key is hidden
        // from, and 0 * inf on the matrix unit would: the weighted values again,
        // key by key over the keys each row sees, against the final reference.
#pragma unroll
        for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[h][e] = f32x4{0, 0, 0, 0};
        pw = load_pages(0);
        for (int i = 0; i < my_steps; ++i) {
            load_k(i);
            f32x4 s;
            (void)scores(i, s);
            const f32x4 p = probs(s);
            const int32_t k0 = k_first + kPage * (wave + NW * i);
            uint32_t nrec;
            const size_t pofs = step_page(i, nrec);
            const __amdgpu_buffer_rsrc_t rv = page_rsrc(vbase, pofs, nrec);
#pragma unroll 1
            for (int t = 0; t < kPage; ++t) {
                const float pt = (t & 2) ? ((t & 1) ? p[3] : p[2]) : ((t & 1) ? p[1] : p[0]);
                const float pk = __shfl(pt, 16 * (t >> 2) + n, 64);
                if (k0 + t < lo || k0 + t >= hi) continue;
                const uint32_t vo = t * row_bytes + (uint32_t)(kvh * D + 16 * grp) * 4u;
#pragma unroll
                for (int h = 0; h < VH; ++h)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {  // dims 64 h + 16 grp + 4 q + e
                        const float4 vv = __builtin_bit_cast(float4, load16_at(rv, vo + 256 * h + 16 * q));
                        o[h][0][q] = fmaf(pk, vv.x, o[h][0][q]);
                        o[h][1][q] = fmaf(pk, vv.y, o[h][1][q]);
                        o[h][2][q] = fmaf(pk, vv.z, o[h][2][q]);
                        o[h][3][q] = fmaf(pk, vv.w, o[h][3][q]);
                    }
            }
        }
    }
    if (page_err && lane == 0) atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);

    // ---- combine the waves: each scales its block to the common reference ------
    l = rg.sum(l);
    if (grp == 0) {
        ml_lds[0][wave][n] = m;
        ml_lds[1][wave][n] = l;
    }
    __syncthreads();
    float mstar = kNegInf, L = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) mstar = fmax_num(mstar, ml_lds[0][w][n]);
    const float mu = mstar == kNegInf ? 0.0f : mstar;
#pragma unroll
    for (int w = 0; w < NW; ++w) L += fast_exp2((ml_lds[0][w][n] - mu) * a.scale_log2) * ml_lds[1][w][n];
    const float scale = fast_exp2((m - mu) * a.scale_log2) * (L > 0.0f ? 1.0f / L : 0.0f);
    if (wave < n_pages) {  // waves without a step hold nothing
#pragma unroll
        for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<f32x4*>(&o_lds[wave][n * D + 64 * h + 16 * grp + 4 * i]) =
                    f32x4{o[h][0][i], o[h][1][i], o[h][2][i], o[h][3][i]} * scale;
    }
    __syncthreads();
    const int nw = min(n_pages, NW);
    for (int e = thread_id(); e < np * (D / 4); e += 64 * NW) {
        f32x4 val = *reinterpret_cast<const f32x4*>(&o_lds[0][4 * e]);
        for (int w = 1; w < nw; ++w) val += *reinterpret_cast<const f32x4*>(&o_lds[w][4 * e]);
        const int r = p0 + e / (D / 4), rq = div_group(a, r);
        const int64_t row = (int64_t)(si.q_start + it.row0 + rq) * a.hq + kvh * G + r - rq * G;
        *reinterpret_cast<f32x4*>(reinterpret_cast<float*>(a.out) + row * D + 4 * (e % (D / 4))) = val;
    }
    if (wave == 0 && grp == 0 && valid)
        a.lse[(int64_t)(si.q_start + qi) * a.hq + head] = L > 0.0f ? fmaf(mstar, a.sm_scale, logf(L)) : kNegInf;
}

// ---------------------------------------------------------------------------
// Merge kernel: one wave per (row, head); combines the partial results of
// split key ranges (and of a shared prefix, for cascade members) by their
// log-sum-exps (lanes over the head dimension).
// ---------------------------------------------------------------------------
template <int D, bool BF16>
__global__ __launch_bounds__(256) void merge_kernel(MArgs a) {
    constexpr int E = D / 64;
    // one row per wave; the wave index is made scalar so that the item is
    // read with scalar loads
    const int idx = wg_id() * 4 + (__builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3);
    const int lane = thread_id() & 63;
    if (idx >= a.n_items) return;
    const MergeItem mi = a.items[idx];
    // slot set 1: slot0 + s * stride, s < nslots (split key ranges of the row's
    // own keys); slot set 2: pad0 + s * pad1, s < pad2 (the chunks of a shared
    // prefix, for cascade members; empty otherwise)
    auto slot_of = [&](int s) -> int64_t {
        return s < mi.nslots ? mi.slot0 + (int64_t)s * mi.stride : mi.pad0 + (int64_t)(s - mi.nslots) * mi.pad1;
    };
    const int n = mi.nslots + mi.pad2;
    // The rows of the first four slots are requested together with the LSEs
    // (their addresses need only the item), so a row with few slots waits for
    // one round trip to memory instead of three.
    float v0[4][E];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int64_t slot = slot_of(u < n ? u : 0);
#pragma unroll
        for (int e = 0; e < E; ++e) v0[u][e] = u < n ? a.part_o[slot * D + lane + 64 * e] : 0.0f;
    }
    // the slots' LSEs are read across the lanes, 64 at a time, and reduced
    // over the wave (a fixed order: the result does not depend on timing)
    float mstar = kNegInf, x0 = kNegInf;
    for (int s0 = 0; s0 < n; s0 += 64) {
        float x = s0 + lane < n ? a.part_lse[slot_of(s0 + lane)] : kNegInf;
        if (s0 == 0) x0 = x;
        for (int off = 32; off > 0; off >>= 1) x = fmaxf(x, __shfl_xor(x, off, 64));
        mstar = fmaxf(mstar, x);
    }
    float acc[E], tot = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
    if (mstar != kNegInf) {
        for (int s0 = 0; s0 < n; s0 += 64) {
            const int cnt = min(64, n - s0);
            // lane j holds the weight of slot s0 + j (the first 64 LSEs are
            // still in registers)
            const float xl = s0 == 0 ? x0 : (lane < cnt ? a.part_lse[slot_of(s0 + lane)] : kNegInf);
            float w = lane < cnt ? expf(xl - mstar) : 0.0f;
            float ws = w;
            for (int off = 32; off > 0; off >>= 1) ws += __shfl_xor(ws, off, 64);
            tot += ws;
            // slots in order; four rows loaded together
            int j = 0;
            if (s0 == 0) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), u));
#pragma unroll
                    for (int e = 0; e < E; ++e)
                        if (u < cnt) acc[e] = fmaf(wj, v0[u][e], acc[e]);
                }
                j = 4;
            }
            for (; j + 4 <= cnt; j += 4) {
                float v[4][E];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int64_t slot = slot_of(s0 + j + u);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[u][e] = a.part_o[slot * D + lane + 64 * e];
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), j + u));
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = fmaf(wj, v[u][e], acc[e]);
                }
            }
            for (; j < cnt; ++j) {
                const int64_t slot = slot_of(s0 + j);
                const float wj = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), j));
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = fmaf(wj, a.part_o[slot * D + lane + 64 * e], acc[e]);
            }
        }
    }
    const float inv = tot > 0.0f ? 1.0f / tot : 0.0f;
    const int64_t row = (int64_t)mi.row * a.hq + mi.head;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float v = acc[e] * inv;
        if (BF16)
            reinterpret_cast<bf16_t*>(a.out)[row * D + lane + 64 * e] = (bf16_t)v;
        else
            reinterpret_cast<float*>(a.out)[row * D + lane + 64 * e] = v;
    }
    if (lane == 0) a.lse[row] = tot > 0.0f ? mstar + logf(tot) : kNegInf;
}

// ---------------------------------------------------------------------------
// KV append: one workgroup per item of up to 16 new rows of one request; wave
// w copies rows w, w + 4, ...  A row is one token's keys (or values) for
// every KV head, contiguous in both the packed input and the page slot, so
// lanes copy it in 16-byte pieces.  A target page outside the pool is
// skipped and sets the error word.
//
// Bound: HBM (5.1 TB/s read + written on 1.3 GB of rows).  NT: stores of a
// small step are non-temporal, so that its rows are in HBM by the time the
// attention streams the cache: left in the memory-side cache, they are written
// back under that stream (256 16-token chunks, 17 MB: append + attention 235 ->
// 225 us; no difference for 3-28 MB before tile work).  A large step's rows are
// better kept there for the attention that reads them next (71 MB: 1705 us
// against 1712 with non-temporal stores, 1.26 GB: 4000 against 4030).
// ---------------------------------------------------------------------------
constexpr int64_t kAppendNtBytes = 32 << 20;
template <bool NT>
__global__ __launch_bounds__(256) void append_kernel(AArgs a) {
    typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
    const WorkItem it = a.items[wg_id()];
    const SeqInfo si = a.seqs[it.seq];
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3, lane = thread_id() & 63;
    const int chunks = a.row_bytes >> 4;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    bool bad = false;
    for (int r = wave; r < it.nrows; r += 4) {
        const int32_t i = it.row0 + r;                 // new row within the request
        const int32_t pos = si.kv_len - si.q_len + i;  // its position in the cache
        const int32_t page = bt_row[pos >> 4];
        if ((uint32_t)page >= (uint32_t)a.num_pages) {
            bad = true;
            continue;
        }
        const int64_t src = (int64_t)(si.q_start + i) * a.row_bytes;
        const int64_t dst = ((int64_t)page * 16 + (pos & 15)) * a.row_bytes;
        const u32x4* ks = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.k_new) + src);
        const u32x4* vs = reinterpret_cast<const u32x4*>(static_cast<const char*>(a.v_new) + src);
        u32x4* kd = reinterpret_cast<u32x4*>(static_cast<char*>(a.k) + dst);
        u32x4* vd = reinterpret_cast<u32x4*>(static_cast<char*>(a.v) + dst);
        for (int c = lane; c < chunks; c += 64) {
            const u32x4 kx = ks[c], vx = vs[c];
            if constexpr (NT) {
                __builtin_nontemporal_store(kx, kd + c);
                __builtin_nontemporal_store(vx, vd + c);
            } else {
                kd[c] = kx;
                vd[c] = vx;
            }
        }
    }
    if (bad && lane == 0) atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);
}

}  // namespace

hipError_t launch_append(const AArgs& a, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    return launch(a.new_bytes <= kAppendNtBytes ? append_kernel<true> : append_kernel<false>, dim3(a.n_items),
                  dim3(256), a, s);
}

namespace {
// both pools within the range of one buffer resource
bool small_pool(const KArgs& a, int head_dim) {
    return (uint64_t)a.num_pages * 16 * a.hkv * head_dim * 2 <= kSmallPoolBytes;
}
template <int MODE, int KS64, int KS128>
hipError_t launch_tile_mode(const KArgs& a, int head_dim, hipStream_t s) {
    const dim3 g((unsigned)a.n_wgs);
    const bool small = small_pool(a, head_dim);
    if (head_dim == 64) {
        const dim3 b(256 * KS64);
        if (small) return launch(tile_kernel<64, 2, kPoolSmall, MODE, 64, KS64>, g, b, a, s);
        else return launch(tile_kernel<64, 2, kPoolLarge, MODE, 64, KS64>, g, b, a, s);
    } else {
        const dim3 b(256 * KS128);
        if (small) return launch(tile_kernel<128, 2, kPoolSmall, MODE, kTileKeysD128, KS128>, g, b, a, s);
        else return launch(tile_kernel<128, 2, kPoolLarge, MODE, kTileKeysD128, KS128>, g, b, a, s);
    }
}
}  // namespace

hipError_t launch_tiles(const KArgs& a, int head_dim, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    // slices need the division's reciprocal; without grouped heads they are the plain rows
    const bool packed = a.group_inv != 0;
    if (a.key_groups)  // as many groups as the plain instance has workgroups per CU
        return packed ? launch_tile_mode<kPacked, 4, 3>(a, head_dim, s) : launch_tile_mode<kRows, 4, 3>(a, head_dim, s);
    return packed ? launch_tile_mode<kPacked, 1, 1>(a, head_dim, s) : launch_tile_mode<kRows, 1, 1>(a, head_dim, s);
}

hipError_t launch_cascade(const KArgs& a, int head_dim, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    return launch_tile_mode<kCascade, 1, 1>(a, head_dim, s);
}

hipError_t launch_few(const KArgs& a, int head_dim, int rb, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    const dim3 g(a.n_items), b(256);
    if (head_dim == 64) {
        if (rb == 1) return launch(few_kernel<64, 1>, g, b, a, s);
        else if (rb == 2) return launch(few_kernel<64, 2>, g, b, a, s);
        else return launch(few_kernel<64, 4>, g, b, a, s);
    } else {  // the planner gives d = 128 units at most 32 rows
        if (rb == 1) return launch(few_kernel<128, 1>, g, b, a, s);
        else return launch(few_kernel<128, 2>, g, b, a, s);
    }
}

hipError_t launch_f32(const KArgs& a, int head_dim, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    if (head_dim == 64)
        return launch(f32_kernel<64, kF32Waves>, dim3(a.n_items), dim3(64 * kF32Waves), a, s);
    else
        return launch(f32_kernel<128, kF32Waves>, dim3(a.n_items), dim3(64 * kF32Waves), a, s);
}

hipError_t scratch_buffer(void** ptr) {
    // the array's device address, looked up once per device with that device
    // current (each GPU holds its own copy at its own address)
    constexpr int kMaxDevices = 64;
    static std::mutex mu;
    static void* addr[kMaxDevices] = {};
    *ptr = nullptr;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= kMaxDevices) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (!addr[dev]) {
        void* p = nullptr;
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess) return e;
        if (!p) return hipErrorInvalidSymbol;
        addr[dev] = p;
    }
    *ptr = addr[dev];
    return hipSuccess;
}

hipError_t launch_merge(const MArgs& a, int head_dim, bool bf16_out, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    const dim3 g((a.n_items + 3) / 4), b(256);
    if (head_dim == 64) {
        if (bf16_out) return launch(merge_kernel<64, true>, g, b, a, s);
        else return launch(merge_kernel<64, false>, g, b, a, s);
    } else {
        if (bf16_out) return launch(merge_kernel<128, true>, g, b, a, s);
        else return launch(merge_kernel<128, false>, g, b, a, s);
    }
}

}  // namespace mstar
