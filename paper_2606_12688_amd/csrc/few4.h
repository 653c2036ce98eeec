// The few-row kernel over a 4-bit cache.
#pragma once
#include "kv4.h"

namespace mstar {
namespace {

// ---------------------------------------------------------------------------
// Few-row attention over a 4-bit cache: the work items, rows and steps of the
// 16-bit few-row kernel (a workgroup is up to 16 RB rows of one KV head, its
// waves take interleaved steps of keys), on other operands.  Both K and V go from
// the pages straight into matrix operands, with nothing through LDS:
//  scores: lane 16 G + n holds dims [G D / 4, +D / 4) of key n, so MFMA step s
//    contracts dims G D / 4 + 8 s .. + 7 of each group G, and Q is read that way;
//  values: the lane holds dims [n D / 16, +D / 16) of keys 4 G .. 4 G + 3, and
//    output row m of block db stands for dim m D / 16 + db.  A conversion gives
//    two dims of one key, an operand register takes two keys of one dim: a byte
//    permute exchanges the halves.
// A lane's share of out is then the D / 4 consecutive dims from G D / 4 on.
//
// Bound: HBM.  Decode steps of 64 requests (28/4 heads, D = 128, 167 MB of cache)
// take 36 us, 4.6 TB/s, of which some 5 us are a workgroup's start; reading their
// pages without computing takes 33.  256 16-token chunks (290 MB) take 76 us, 3.8
// TB/s; reading alone 69, computing alone 55.  A step's registers take the next step's loads as
// soon as they are read; larger steps (64 keys) or two and three steps in flight
// change nothing (decode 42-46 us with its merge, chunks 82-99), but loads in a
// branch, which the compiler cannot count and waits for together, cost the
// chunks 92 us for 82.  Non-temporal loads of the codes: 51 -> 46 us for 128
// decode steps behind a shared prefix.
// ---------------------------------------------------------------------------
template <int D, int RB, int NW>  // NW waves
struct Few4Lds {
    static constexpr int PC = D / 16;         // 16-byte pieces of a lane's results per row block
    static constexpr bool QLDS = RB * D >= 256;  // Q in LDS: in registers it would cost a wave per SIMD
    // a wave's results while they are combined; before that, Q
    static constexpr int kBytes = NW * PC * 64 * 16;
    static_assert(!QLDS || RB * (D / 32) * 64 * 16 <= kBytes, "Q fits where the results go");
    struct Stats {
        float ml[NW][2][RB * 16];
        float fin[2][RB * 16];
    };
};

// Work item `item` of the launch; `lds` has Few4Lds::kBytes, 16-byte aligned.
template <int D, int RB, int NW>
__device__ __forceinline__ void few4_item(const KArgs& a, int item, char* lds, typename Few4Lds<D, RB, NW>::Stats& stats) {
    typedef Record<D> R;
    typedef Few4Lds<D, RB, NW> L4;
    constexpr int PC = L4::PC;
    constexpr bool QLDS = L4::QLDS;
    constexpr int PG = 2, SK = 16 * PG;  // pages and keys of a step
    constexpr int DS = D / 32, DB = D / 16;
    constexpr int NC = D / 32;         // dwords of codes per lane and record
    f32x4 (*o_lds)[PC * 64] = reinterpret_cast<f32x4 (*)[PC * 64]>(lds);
    bf16x8 (*q_lds)[DS][64] = reinterpret_cast<bf16x8 (*)[DS][64]>(lds);
    auto& ml_lds = stats.ml;
    auto& fin_lds = stats.fin;

    const WorkItem it = a.items[item];
    const int tid = thread_id(), wave = __builtin_amdgcn_readfirstlane(tid >> 6) & (NW - 1), lane = tid & 63;
    const int n = lane & 15, grp = lane >> 4;
    const int G = a.group;
    const int kvh = it.head;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    const RowGroup rg;

    // Step i of this wave starts at key k_begin + SK (wave + NW i) and spans PG
    // pages; the page indices of 64 / PG steps live in one register (lane PG i + h
    // holds page h of step i), the next window's in another.
    constexpr int WS = 64 / PG;  // steps per window
    const int n_steps = (it.k_end - it.k_begin + SK - 1) / SK;
    const int my_steps = wave < n_steps ? (n_steps - wave + NW - 1) / NW : 0;
    const int32_t page0 = it.k_begin >> 4;
    const int32_t n_pages = ((it.k_end + 15) >> 4) - page0;
    auto load_pages = [&](int first_step) {
        const int i = first_step + lane / PG, pg = PG * (wave + NW * i) + lane % PG;
        return i < my_steps && pg < n_pages ? bt_row[page0 + pg] : -1;
    };
    int32_t pw_cur = load_pages(0), pw_next = my_steps > WS ? load_pages(WS) : -1;
    const char* kbase = reinterpret_cast<const char*>(a.k);
    const char* vbase = reinterpret_cast<const char*>(a.v);
    const int koff = R::kScales + (grp * (D / 4) / 32) * 16 + n, voff = R::scale(4 * grp, n);
    bool page_err = false;
    // this lane's codes of a step's records, and its scale bytes: one for its key
    // (K), one for each of its four keys (V)
    uint32_t kc[PG][NC], vc[PG][NC], ks[PG], vs[PG];
    __amdgpu_buffer_rsrc_t rv[PG];
    auto load_codes = [&](__amdgpu_buffer_rsrc_t r, uint32_t (&x)[NC]) {
        if constexpr (D == 128) {
            const uint4 c = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, lane * 16, 0, kCachePolicyNT));
            x[0] = c.x; x[1] = c.y; x[2] = c.z; x[3] = c.w;
        } else {
            typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
            const u32x2 c = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, lane * 8, 0, kCachePolicyNT));
            x[0] = c[0]; x[1] = c[1];
        }
    };
    // Pages outside the pool, past the item's end and of steps behind the last read
    // zeros through an empty buffer range: no load sits in a branch, where the
    // compiler could not count it and would wait for all loads before each use.
    auto load_k = [&](int i) {  // also names the step's V records, for load_v
        if (i > 0 && i % WS == 0) {
            pw_cur = pw_next;
            pw_next = i + WS < my_steps ? load_pages(i + WS) : -1;
        }
#pragma unroll
        for (int h = 0; h < PG; ++h) {
            const int32_t page = __builtin_amdgcn_readlane(pw_cur, PG * (i % WS) + h);
            const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
            page_err |= !ok && i < my_steps && PG * (wave + NW * i) + h < n_pages;
            const size_t ofs = ok ? ((size_t)page * a.hkv + kvh) * R::kBytes : 0;
            const uint32_t nrec = ok ? (uint32_t)R::kBytes : 0u;
            const __amdgpu_buffer_rsrc_t rk = page_rsrc(kbase, ofs, nrec);
            rv[h] = page_rsrc(vbase, ofs, nrec);
            load_codes(rk, kc[h]);
            ks[h] = __builtin_amdgcn_raw_buffer_load_b8(rk, koff, 0, 0);
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int h = 0; h < PG; ++h) {
            load_codes(rv[h], vc[h]);
            vs[h] = __builtin_amdgcn_raw_buffer_load_b32(rv[h], voff, 0, 0);
        }
    };
    // the first step's loads go out before anything that waits: a workgroup's
    // start is a chain of reads (item, page indices, pages)
    load_k(0);
    load_v();

    const SeqInfo si = a.seqs[it.seq];
    int32_t lo[RB], hi[RB];
    bf16x8 q_reg[QLDS ? 1 : RB][DS];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = rb * 16 + n;
        const bool valid = r < it.nrows;
        const int rr = it.row0 + r;
        const int qi = div_group(a, rr), h = kvh * G + rr - qi * G;
        lo[rb] = 0;
        hi[rb] = 0;
        if (valid) row_interval(a, si, it, qi, lo[rb], hi[rb]);
        const int64_t qoff = ((int64_t)(si.q_start + qi) * a.hq + h) * D + grp * (D / 4);
        if constexpr (QLDS) {
            for (int s = wave; s < DS; s += NW)
                q_lds[rb][s][lane] = valid ? __builtin_bit_cast(bf16x8, load16(a.q, qoff + 8 * s)) : bf16x8{};
        } else {
#pragma unroll
            for (int s = 0; s < DS; ++s)
                q_reg[rb][s] = valid ? __builtin_bit_cast(bf16x8, load16(a.q, qoff + 8 * s)) : bf16x8{};
        }
    }
    if constexpr (QLDS) __syncthreads();
    auto qf = [&](int rb, int s) -> bf16x8 {
        if constexpr (QLDS) return q_lds[rb][s][lane];
        else return q_reg[rb][s];
    };
    int32_t lo_max, hi_min, dummy;
    {
        const int q_first = div_group(a, it.row0), q_last = div_group(a, it.row0 + it.nrows - 1);
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

    auto compute_step = [&](int i) {
        const int32_t k0 = it.k_begin + SK * (wave + NW * i);
        f32x4 sc[RB][PG];
#pragma unroll
        for (int h = 0; h < PG; ++h) {
            const float sk = scale_of(ks[h]);
#pragma unroll
            for (int s = 0; s < DS; ++s) {
                const bf16x8 kf = eight_of(kc[h][s], sk);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) sc[rb][h] = mfma16(kf, qf(rb, s), s == 0 ? f32x4{0, 0, 0, 0} : sc[rb][h]);
            }
            if constexpr (RB > 1) __builtin_amdgcn_sched_barrier(0);
        }
        load_k(i + 1);  // the K registers are free
        if (!(k0 >= lo_max && k0 + SK <= hi_min)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                const int32_t lo_r = lo[rb] - (k0 + 4 * grp), hi_r = hi[rb] - (k0 + 4 * grp);
#pragma unroll
                for (int h = 0; h < PG; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int c = h * 16 + e;
                        if (!(c >= lo_r && c < hi_r)) sc[rb][h][e] = kNegInf;
                    }
            }
        }
        float alpha[RB];
        if (softmax_lazy<RB, PG>(rg, sc, a.scale_log2, m, l, alpha)) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int db = 0; db < DB; ++db) o[rb][db] *= alpha[rb];
        }
#pragma unroll
        for (int c = 0; c < PG / 2; ++c) {  // 32 keys of the value product
            bf16x8 pf[RB];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) pf[rb] = to_bf16x8(sc[rb][2 * c], sc[rb][2 * c + 1]);
            float sv[2][4];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int j = 0; j < 4; ++j) sv[h][j] = scale_of(v_scale(vs[2 * c + h], j));
#pragma unroll
            for (int b = 0; b < DB / 2; ++b) {  // dims 2 b and 2 b + 1 of the lane's: blocks 2 b and 2 b + 1
                uint32_t even[4], odd[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t y[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        y[j] = __builtin_bit_cast(uint32_t, v_pair<D>(vc[2 * c + h], j, b, sv[h][j]));
                    even[2 * h] = __builtin_amdgcn_perm(y[1], y[0], 0x05040100);
                    even[2 * h + 1] = __builtin_amdgcn_perm(y[3], y[2], 0x05040100);
                    odd[2 * h] = __builtin_amdgcn_perm(y[1], y[0], 0x07060302);
                    odd[2 * h + 1] = __builtin_amdgcn_perm(y[3], y[2], 0x07060302);
                }
                const bf16x8 ve = __builtin_bit_cast(bf16x8, uint4{even[0], even[1], even[2], even[3]});
                const bf16x8 vo = __builtin_bit_cast(bf16x8, uint4{odd[0], odd[1], odd[2], odd[3]});
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    o[rb][2 * b] = mfma16(ve, pf[rb], o[rb][2 * b]);
                    o[rb][2 * b + 1] = mfma16(vo, pf[rb], o[rb][2 * b + 1]);
                }
                if constexpr (RB > 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        load_v();  // the V registers are free
    };

    for (int i = 0; i < my_steps; ++i) compute_step(i);
    if (page_err && lane == 0) atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);

    // ---- combine the waves ------------------------------------------------------
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float lt = rg.sum(l[rb]);
        if (grp == 0) {
            ml_lds[wave][0][rb * 16 + n] = m[rb];
            ml_lds[wave][1][rb * 16 + n] = lt;
        }
    }
    __syncthreads();
    // one row block at a time: each wave leaves its results against the common
    // reference, 16-byte pieces in lane order, and all threads add them up
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
        if (rb > 0) __syncthreads();  // the previous block has been added up
#pragma unroll
        for (int p = 0; p < PC; ++p) {  // dims G D / 4 + 4 p ..: row r of blocks db .. db + 3
            const int r = 4 * p / DB, db = 4 * p % DB;
            o_lds[wave][p * 64 + lane] = f32x4{o[rb][db][r], o[rb][db + 1][r], o[rb][db + 2][r], o[rb][db + 3][r]} * own;
        }
        __syncthreads();
        for (int e = tid; e < PC * 64; e += 64 * NW) {
            const int r = rb * 16 + (e & 15), d4 = ((e >> 4) & 3) * (D / 4) + 4 * (e >> 6);
            if (r >= it.nrows) continue;
            f32x4 val = o_lds[0][e];
#pragma unroll
            for (int w = 1; w < NW; ++w) val += o_lds[w][e];
            const float L = fin_lds[1][r];
            val *= L > 0.0f ? __builtin_amdgcn_rcpf(L) : 0.0f;  // off by one ulp of fp32 at most
            const float lse = L > 0.0f ? (fin_lds[0][r] + __log2f(L)) * kLn2 : kNegInf;
            const int rr = it.row0 + r, qi = div_group(a, rr);
            if (it.part < 0) {
                const int64_t orow = (int64_t)(si.q_start + qi) * a.hq + kvh * G + rr - qi * G;
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

template <int D, int RB, int NW>
__global__ __launch_bounds__(64 * NW, RB == 1 ? 4 : (RB == 2 ? 3 : 2)) void few4_kernel(KArgs a) {
    __shared__ __attribute__((aligned(1024))) char lds[Few4Lds<D, RB, NW>::kBytes];
    __shared__ typename Few4Lds<D, RB, NW>::Stats stats;
    few4_item<D, RB, NW>(a, wg_id(), lds, stats);
}

}  // namespace
}  // namespace mstar
