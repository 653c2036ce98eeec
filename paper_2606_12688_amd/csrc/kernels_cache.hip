// HIP kernels of the operators on paged caches (mstar_cache.h) for gfx950: the
// 4-bit cache's append, attention and read-back, and block tables.
#include "kv4.h"

namespace mstar {
namespace {

// ---------------------------------------------------------------------------
// Append: a workgroup takes up to 16 new rows of one request, a wave one KV head
// of the rows of one aligned group of four positions at a time: lane 4 n + j holds
// dims [n D / 16, +D / 16) of the group's key j, so that its V words are
// consecutive and its K words run over 64 (D = 128) or 32 bytes of each piece.
// The 32 dims of a scale are 4 (D = 128) or 8 neighbouring n.
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void append4_kernel(Append4Args a) {
    constexpr int E = D / 16;  // dims per lane
    typedef Record<D> R;
    const WorkItem it = a.items[wg_id()];
    const SeqInfo si = a.seqs[it.seq];
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3, lane = thread_id() & 63;
    const int n = lane >> 2, j = lane & 3;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    const int32_t g0 = it.k_begin >> 2, groups = ((it.k_end - 1) >> 2) - g0 + 1;
    bool bad_page = false, bad_value = false;
    for (int t = wave; t < groups * a.hkv; t += 4) {
        const int g = t / a.hkv, head = t - g * a.hkv;
        const int32_t pos = 4 * (g0 + g) + j, slot = pos & 15;
        bool live = pos >= it.k_begin && pos < it.k_end;
        const int32_t page = live ? bt_row[pos >> 4] : 0;
        if ((uint32_t)page >= (uint32_t)a.num_pages) {
            bad_page = true;
            live = false;
        }
        const int64_t row = si.q_start + (pos - (si.kv_len - si.q_len));
        const int64_t src = (row * a.hkv + head) * D + n * E;
        const int64_t rec = ((int64_t)page * a.hkv + head) * R::kBytes;
#pragma unroll
        for (int m = 0; m < 2; ++m) {  // K, V
            uint32_t x[E];
            const uint16_t* in = reinterpret_cast<const uint16_t*>(m == 0 ? a.k_new : a.v_new) + src;
            uint32_t top = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[e] = live ? in[e] : 0;
                bad_value |= (x[e] & 0x7fff) >= 0x7f80;
                if ((x[e] & 0x7fff) > 0x7f80) x[e] = 0;
                top = max(top, x[e] & 0x7fff);
            }
            // the largest magnitude of the scale's 32 dims
            top = max(top, (uint32_t)__shfl_xor((int)top, 4, 64));
            top = max(top, (uint32_t)__shfl_xor((int)top, 8, 64));
            if (D == 64) top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
            // smallest b with top <= 7 * 2^(b - 127): 7 is mantissa 0x60 two binades up
            const int b = min(max((int)((top + 31) >> 7) - 2, kScaleMin), kScaleMax);
            const float inv = __uint_as_float((uint32_t)(254 - b) << 23);  // exact
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float y = __uint_as_float((x[e] & 0x7fff) << 16) * inv;
                // nearest of 0, .5, 1, 1.5, 2, 3, 4, 6, ties to the even code
                const uint32_t c = (y > 0.25f) + (y >= 0.75f) + (y > 1.25f) + (y >= 1.75f) + (y > 2.5f) +
                                   (y >= 3.5f) + (y > 5.0f);
                w |= (c | (x[e] >> 15) << 3) << (4 * e);
            }
            if (!live) continue;
            char* to = static_cast<char*>(m == 0 ? a.k : a.v) + rec;
            char* word = to + (m == 0 ? R::k_word(slot, n) : R::v_word(slot, n));
            if (D == 128)
                *reinterpret_cast<uint32_t*>(word) = w;
            else
                *reinterpret_cast<uint16_t*>(word) = (uint16_t)w;
            if (n % (32 / E) == 0) to[R::scale(slot, n)] = (char)b;
        }
    }
    const int bits = (__builtin_amdgcn_ballot_w64(bad_page) ? MSTAR_DEVERR_PAGE_RANGE_BIT : 0) |
                     (__builtin_amdgcn_ballot_w64(bad_value) ? MSTAR_DEVERR_NONFINITE_BIT : 0);
    if (bits && lane == 0) atomicOr(a.err, bits);
}

// ---------------------------------------------------------------------------
// Unpack: a wave takes one record of a listed page, four keys at a time; lane
// 16 g + n writes dims [n D / 16, +D / 16) of the group's key g.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void store_word(bf16_t* out, uint32_t w, float s) {
    const bf16x2 p0 = pair_of<0>(w, s), p1 = pair_of<1>(w, s);
    if constexpr (D == 128) {
        const bf16x2 p2 = pair_of<2>(w, s), p3 = pair_of<3>(w, s);
        *reinterpret_cast<bf16x8*>(out) = bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
    } else {
        *reinterpret_cast<bf16x4*>(out) = bf16x4{p0[0], p0[1], p1[0], p1[1]};
    }
}

template <int D>
__global__ __launch_bounds__(256) void unpack4_kernel(Unpack4Args a) {
    typedef Record<D> R;
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3, lane = thread_id() & 63;
    const int g = lane >> 4, n = lane & 15;
    const int64_t task = (int64_t)wg_id() * 4 + wave;
    if (task >= (int64_t)a.n_ids * a.hkv) return;
    const int64_t i = task / a.hkv;
    const int head = (int)(task - i * a.hkv);
    const int32_t page = a.ids[i];
    const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
    const int64_t rec = ok ? ((int64_t)page * a.hkv + head) * R::kBytes : 0;
#pragma unroll
    for (int m = 0; m < 2; ++m) {
        const unsigned char* from = static_cast<const unsigned char*>(m == 0 ? a.k : a.v) + rec;
        bf16_t* out = static_cast<bf16_t*>(m == 0 ? a.k_out : a.v_out);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int slot = 4 * c + g;
            uint32_t w = 0, b = 0;
            if (ok) {
                const unsigned char* word = from + (m == 0 ? R::k_word(slot, n) : R::v_word(slot, n));
                w = D == 128 ? *reinterpret_cast<const uint32_t*>(word) : *reinterpret_cast<const uint16_t*>(word);
                b = from[R::scale(slot, n)];
            }
            store_word<D>(out + ((i * 16 + slot) * a.hkv + head) * D + n * (D / 16), w, scale_of(b));
        }
    }
}

// ---------------------------------------------------------------------------
// Attention: a wave per (query row, head), a page at a time.  Lane 16 G + n
// forms its share of key n's score (dims [G D / 4, +D / 4)) and of the values of
// keys 4 G .. 4 G + 3 (dims [n D / 16, +D / 16)).
// ---------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void rows4_kernel(KArgs a) {
    constexpr int EK = D / 4, EV = D / 16;
    typedef Record<D> R;
    const int item = wg_id() / a.hq, head = wg_id() - item * a.hq;
    const WorkItem it = a.items[item];
    const SeqInfo si = a.seqs[it.seq];
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3, lane = thread_id() & 63;
    const int n = lane & 15, grp = lane >> 4;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    bool page_err = false;
    for (int r = wave; r < it.nrows; r += 4) {
        const int i = it.row0 + r;
        const int32_t pos = si.kv_len - si.q_len + i;
        const int32_t lo = si.window > 0 ? max(0, pos - si.window + 1) : 0, hi = a.row_hi[si.hi_off + i];
        const int64_t row = (int64_t)(si.q_start + i) * a.hq + head;
        float q[EK];
#pragma unroll
        for (int e = 0; e < EK; ++e) q[e] = (float)static_cast<const bf16_t*>(a.q)[row * D + grp * EK + e];
        float m = kNegInf, l = 0.0f, o[EV];
#pragma unroll
        for (int e = 0; e < EV; ++e) o[e] = 0.0f;
        for (int32_t k0 = lo & ~15; k0 < hi; k0 += 16) {
            const int32_t page = bt_row[k0 >> 4];
            const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
            page_err |= !ok;
            const int64_t rec = ok ? ((int64_t)page * a.hkv + head / a.group) * R::kBytes : 0;
            const unsigned char* kr = static_cast<const unsigned char*>(a.k) + rec;
            const unsigned char* vr = static_cast<const unsigned char*>(a.v) + rec;
            float s = 0.0f;
#pragma unroll
            for (int d = 0; d < EK / 8; ++d) {
                const uint32_t w = ok ? reinterpret_cast<const uint32_t*>(kr)[lane * (D / 32) + d] : 0;
                const float sc = scale_of(ok ? kr[R::scale(n, 4 * grp)] : 0);
                const bf16x2 p0 = pair_of<0>(w, sc), p1 = pair_of<1>(w, sc), p2 = pair_of<2>(w, sc), p3 = pair_of<3>(w, sc);
                s += q[8 * d] * (float)p0[0] + q[8 * d + 1] * (float)p0[1] + q[8 * d + 2] * (float)p1[0] +
                     q[8 * d + 3] * (float)p1[1] + q[8 * d + 4] * (float)p2[0] + q[8 * d + 5] * (float)p2[1] +
                     q[8 * d + 6] * (float)p3[0] + q[8 * d + 7] * (float)p3[1];
            }
            s += __shfl_xor(s, 16, 64);
            s += __shfl_xor(s, 32, 64);
            if (k0 + n < lo || k0 + n >= hi) s = kNegInf;
            float top = s;
            for (int x = 8; x > 0; x >>= 1) top = fmax_num(top, __shfl_xor(top, x, 64));
            const float m_new = fmax_num(m, top * a.scale_log2);
            const float alpha = fast_exp2(m - m_new);
            m = m_new;
            const float p = fast_exp2(fmaf(s, a.scale_log2, -m));
            l = l * alpha + p;
#pragma unroll
            for (int e = 0; e < EV; ++e) o[e] *= alpha;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int slot = 4 * grp + j;
                const float pj = __shfl(p, slot, 64);
                uint32_t w = 0, b = 0;
                if (ok) {
                    const unsigned char* word = vr + R::v_word(slot, n);
                    w = D == 128 ? *reinterpret_cast<const uint32_t*>(word) : *reinterpret_cast<const uint16_t*>(word);
                    b = min((int)vr[R::scale(slot, n)], kScaleMax);
                }
                const float sc = scale_of(b);
                const bf16x2 v[4] = {pair_of<0>(w, sc), pair_of<1>(w, sc), pair_of<2>(w, sc), pair_of<3>(w, sc)};
#pragma unroll
                for (int e = 0; e < EV; ++e) o[e] = fmaf(pj, (float)v[e >> 1][e & 1], o[e]);
            }
        }
        for (int x = 8; x > 0; x >>= 1) l += __shfl_xor(l, x, 64);
#pragma unroll
        for (int e = 0; e < EV; ++e) {
            o[e] += __shfl_xor(o[e], 16, 64);
            o[e] += __shfl_xor(o[e], 32, 64);
            o[e] *= l > 0.0f ? 1.0f / l : 0.0f;
            if (grp == 0) static_cast<bf16_t*>(a.out)[row * D + n * EV + e] = (bf16_t)o[e];
        }
        if (lane == 0) a.lse[row] = l > 0.0f ? (m + __log2f(l)) * kLn2 : kNegInf;
    }
    if (page_err && lane == 0) atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);
}

// ---------------------------------------------------------------------------
// Block tables: a thread per new row.  The row that starts a page enters it; rows
// of one page read the same entry of the free list, so no thread waits for
// another.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(256) void tables_kernel(TablesArgs a) {
    const int item = wg_id() * 16 + (thread_id() >> 4), r = thread_id() & 15;
    if (item >= a.n_items) return;
    const WorkItem it = a.items[item];
    if (r >= it.nrows) return;
    const SeqInfo si = a.seqs[it.seq];
    const int32_t first = si.kv_len - si.q_len;  // cached positions
    const int32_t pos = it.k_begin + r, entry = pos >> 4, held = (first >> 4) + ((first & 15) != 0);
    int32_t* bt = a.bt + (int64_t)it.seq * a.bt_stride + entry;
    const bool taken = entry >= held;
    int32_t page = taken ? a.free_pages[si.page_off + (entry - held)] : *bt;
    if ((uint32_t)page >= (uint32_t)a.num_pages) {
        page = -1;
        atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);
    }
    if (taken && (pos & 15) == 0) *bt = page;
    if (a.slots) a.slots[si.q_start + it.row0 + r] = page < 0 ? -1 : (int64_t)page * 16 + (pos & 15);
}

}  // namespace

hipError_t launch_append4(const Append4Args& a, int head_dim, hipStream_t s) {
    return launch(head_dim == 64 ? append4_kernel<64> : append4_kernel<128>, dim3(a.n_items), dim3(256), a, s);
}

hipError_t launch_unpack4(const Unpack4Args& a, int head_dim, hipStream_t s) {
    const int64_t wgs = ((int64_t)a.n_ids * a.hkv + 3) / 4;
    if (wgs > INT32_MAX) return hipErrorInvalidValue;
    return launch(head_dim == 64 ? unpack4_kernel<64> : unpack4_kernel<128>, dim3((unsigned)wgs), dim3(256), a, s);
}

hipError_t launch_rows4(const KArgs& a, int head_dim, hipStream_t s) {
    const dim3 g((unsigned)a.n_items * (unsigned)a.hq);
    return launch(head_dim == 64 ? rows4_kernel<64> : rows4_kernel<128>, g, dim3(256), a, s);
}

hipError_t launch_tables(const TablesArgs& a, hipStream_t s) {
    return launch(tables_kernel, dim3((a.n_items + 15) / 16), dim3(256), a, s);
}

}  // namespace mstar
