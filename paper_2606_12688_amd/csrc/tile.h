// The multi-row tile kernel, over a 16-bit or a 4-bit cache.
#pragma once
#include <type_traits>

#include "device.h"
#include "few4.h"

namespace mstar {
namespace {

// ---------------------------------------------------------------------------
// Multi-row tile kernel: one workgroup = 64 * RBW query rows of one query head
// (4 waves x RBW blocks of 16 rows) against the item's key range, 64 keys per
// tile, K and V tiles double-buffered in LDS.
//
// K/V tiles go from HBM straight into LDS (buffer loads with the LDS bit: lane
// i of a wave writes bytes [16 i, 16 i + 16) after the wave's base address), so
// no VGPRs, no LDS store instructions and no wait for the data sit between a
// tile's load and its use.  Rows are stored unpadded (2 D bytes) and the
// 16-byte chunks of each row are XOR-permuted by a function of the row, chosen
// so that the lanes served together by the K fragment reads (16 rows, one
// chunk column) and by the transposing V reads (8 rows, 32 bytes each) hit
// distinct banks.  The permutation is applied on the load side: the lane that
// fills physical chunk p of row r fetches logical chunk p ^ swz(r).
// ---------------------------------------------------------------------------
// Keys per tile of the d = 128 tile kernel: 32-key tiles (32 KB of LDS, 162
// VGPRs) run three workgroups per CU instead of two with 64-key tiles, which
// the extra barrier per 32 keys more than pays for (text+latent 1.788 ->
// 1.713 ms, CFG labels 2.120 -> 2.006 ms).  At d = 64 the 64-key tile stays:
// 32-key tiles at five workgroups per CU were 1.6% slower.
#ifndef MSTAR_TILE_KEYS_D128
#define MSTAR_TILE_KEYS_D128 32
#endif
constexpr int kTileKeysD128 = MSTAR_TILE_KEYS_D128;

// Occupancy: two workgroups per CU at d = 128 with 64-key tiles (64 KB of
// LDS and up to 256 VGPRs each), four at d = 64 (32 KB, at most 128 VGPRs: the
// softmax's vector work, which bounds d = 64, then has four waves per SIMD to
// draw from).  BN keys per tile: 64, or 32 (half the LDS and score registers
// for a third workgroup per CU at d = 128, with a barrier per 32 keys).
// KS > 1: KS groups of four waves take a run of the workgroup's tiles each, with
// tile buffers of their own, and their results are added up in LDS at the end.
// For launches that leave a CU at most one workgroup: it then has as many waves
// as KS workgroups would give it, on a KS-th of the keys.
// 4-bit tiles at d = 64 hold more addresses than 128 VGPRs take: 2-4 registers spill
// (mixed launches, FEW below: 4 in a cascade, 9 packed, 12 by rows; by rows at d =
// 128 with 32 keys 4), and a reload in the loop waits for the tile ahead's loads too.
// At three waves per SIMD nothing spills, and either wins, us with four -> three:
// four prompts of 2000 tokens, 16/8 heads, 84 -> 71, 16 of 1000 69 -> 72, two of
// 6000 165 -> 185, 28/4 heads 267 -> 273; 16 rollouts 164 -> 169, 28/4 241 -> 250;
// mixed, 48 decode steps beside a prompt of 1000, 16/8, 36.5 -> 32.3, 32 beside two
// of 2000 65 -> 59, 16 beside 16 rollouts, 28/4, 250 -> 258.
//
// How a workgroup's rows are named: query rows of one head, (query row, head)
// pairs of a KV head's group, or entries of a cascade's row list.
enum { kRows, kPacked, kCascade };

// What it reads: a 16-bit pool of up to 2 GB or of any size, or a 4-bit pool.
//
// A 4-bit tile cannot go straight into LDS: a wave loads its share (of two pages the
// 16 keys of one, K or V; of four, both of one) into registers a tile ahead, a lane
// its D / 8 bytes of each record, and converts them into the same LDS image that
// the direct loads of a 16-bit tile leave, so that each value is converted once
// per workgroup and everything after it is the same.  Bound as the 16-bit instances
// are (vector issue beside the matrix units), with the conversions on top, and at D =
// 64 LDS bank conflicts of the converted V (26 of a rollout's us).  In turn on one
// card, on the same values, us with 16 -> 4 bits: eight requests of 256 + 4096 tokens,
// 28/4 heads at D = 128, 1613 -> 1762 (1160 TFLOP/s); 64 rollouts of 768 rows at D = 64
// 520 -> 588; four prompts of 200-2000 tokens 56 -> 59.
enum { kPoolSmall, kPoolLarge, kPool4 };

// FEW > 0: the launch also holds the few-row items of a 4-bit cache, of FEW 16-row
// blocks, in workgroups of their own behind the tiles': they stream from memory
// while the last tiles keep the matrix units busy, without a side stream's fork
// and join, at the tiles' occupancy.  128 decode steps behind a shared prefix 42.5
// -> 34 us; 48 decode steps beside a prompt of 1000 tokens 52 -> 44, beside 64
// chunks and an image of 4352 319 -> 310; 96 beside four prompts of 2500 and the
// image 520 -> 491.  Spread evenly among the tiles instead, they took up to 50%
// longer (a prompt's last tiles start late).  At d = 64, with the side stream -> in one
// launch: 48 decode steps and a prompt of 1000 tokens, 16/8 heads, 48 -> 36.5 us, 28/4
// 43.4 -> 34.2; 100 and four of 2000 108 -> 94, 28/4 123 -> 108; 4 and one of 1000, 28/4,
// 38 either way; 16 and 16 rollouts 172 -> 165.
__device__ __forceinline__ const KArgs& tile_args(const KArgs& a) { return a; }
__device__ __forceinline__ const KArgs& tile_args(const MixedArgs& a) { return a.tile; }

template <int D, int RBW, int CACHE, int MODE, int BN, int KS, int FEW = 0>
__global__ __launch_bounds__(256 * KS, CACHE == kPool4 && KS > 1 ? KS : D == 64 ? 4 : (BN == 32 ? 3 : 2)) void tile_kernel(
    std::conditional_t<FEW == 0, KArgs, MixedArgs> args) {
    const KArgs& a = tile_args(args);
    static_assert(BN == 32 || BN == 64, "tile sizes");
    constexpr int NW = 4;            // waves per key group (32 rows each)
    constexpr int NB = BN / 16;      // 16-key blocks of a tile
    constexpr int NC = BN / 32;      // 32-key steps of the value product
    constexpr int RBY = 2 * D;       // bytes per K/V row in LDS
    constexpr int CH = D / 8;        // 16-byte chunks per row
    constexpr int DS = D / 32;       // MFMA steps over the head dimension
    constexpr int DB = D / 16;       // 16-wide blocks of O^T
    constexpr int NLD = BN * CH / (64 * NW);  // direct loads per wave, matrix and tile
    constexpr int RPL = 64 / CH;     // rows filled by one wave-wide load
    constexpr int TB = BN * RBY;     // bytes of one K or V tile
    constexpr int PPT = BN / 16;     // pages per tile
    constexpr bool SMALL = CACHE == kPoolSmall;
    static_assert(CACHE != kPool4 || (PPT == NW / 2 && D == 128) || PPT == NW, "shares of a 4-bit tile");
    // two tile buffers per key group ([K, V] of its even and odd tiles): tile
    // t + 1 loads into one while tile t is read from the other
    __shared__ __attribute__((aligned(1024))) char bufs[2][KS][2][TB];
    __shared__ __attribute__((aligned(256))) int32_t page_rings[CACHE == kPool4 ? 1 : KS][2][64];
    // each row's visible interval [lo, hi), read on partial tiles only (kept
    // out of the registers the tile loop carries)
    __shared__ __attribute__((aligned(16))) int2 row_lohi[NW][16 * RBW];

    const int wg = wg_id();
    if constexpr (FEW > 0) {
        typedef Few4Lds<D, FEW, NW> F;
        static_assert(KS == 1 && F::kBytes <= (int)sizeof(bufs), "few-row items use the tile buffers");
        __shared__ typename F::Stats stats;
        if (wg >= a.n_wgs) {
            if (wg - a.n_wgs < args.few.n_items) few4_item<D, FEW, NW>(args.few, wg - a.n_wgs, &bufs[0][0][0][0], stats);
            return;
        }
    }

    // The planner's launch order names the (item, query head) of every
    // workgroup; it keeps the workgroups that read the same K/V pages on one
    // XCD.  Padding entries (item < 0) exit.
    const int item = a.order[2 * wg], head = a.order[2 * wg + 1];
    if (item < 0) return;
    const int kvh = head / a.group;
    const WorkItem it = a.items[item];
    const SeqInfo si = a.seqs[it.seq];
    // Rows of this workgroup: np (query row, head) pairs from pair p0 on, g
    // heads from head0 on per query row.  A full item gives each head's rows a
    // workgroup.  The G workgroups of an item that is not full (a request's last
    // rows, or all of a short one) share its nrows * G pairs out, query row
    // first, as slices of 64 RBW, the last of which have nothing to do: a
    // 16-token chunk of 7 heads per KV head fills one slice instead of 16 of
    // 128 rows in each of seven (48 decode steps, 64 such chunks, one image and
    // 16 rollouts in one launch: 687 -> 617 us).  Full items keep one head each:
    // sharing them out as well changes nothing where every row sees the same
    // keys and costs 2% on causal prompts.  A cascade item names its rows itself.
    int p0 = 0, np = it.nrows, g = 1, head0 = head;
    if (MODE == kPacked && it.nrows < 64 * RBW) {
        g = a.group;
        head0 = kvh * g;
        p0 = (head - head0) * 64 * RBW;
        np = min(it.nrows * g - p0, 64 * RBW);
        if (np <= 0) return;
    }
    auto query_of = [&](int p) -> int {  // query row of pair p: p / g (exact, see group_inv)
        return MODE != kPacked || g == 1 ? p : (int)(((uint64_t)(uint32_t)p * a.group_inv) >> 32);
    };
    // the wave index is wave-uniform; readfirstlane lets the compiler keep
    // everything derived from it (row bounds, loop decisions) in scalars
    const int tid = thread_id(), lane = tid & 63;
    const int wave_all = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wave = wave_all & (NW - 1), kg = KS == 1 ? 0 : wave_all / NW;  // wave within its key group, and the group
    char (&buf0)[2][TB] = bufs[0][kg];
    char (&buf1)[2][TB] = bufs[1][kg];
    int32_t (&page_ring)[2][64] = page_rings[CACHE == kPool4 ? 0 : kg];
    const int n = lane & 15, grp = lane >> 4;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    const RowGroup rg;

    // ---- rows owned by this lane ------------------------------------------
    // kCascade (a shared-prefix cascade item): row r is entry row0 + r of the row
    // list, a (packed query row, query head) of some group member; every key
    // of the item is visible to it.
    int32_t lo[RBW], hi[RBW];  // written to row_lohi, read back on partial tiles
    bool valid[RBW];
    bf16x8 qf[RBW][DS];
#pragma unroll
    for (int rb = 0; rb < RBW; ++rb) {
        const int r = wave * 16 * RBW + rb * 16 + n;
        valid[rb] = r < np;
        lo[rb] = 0;
        hi[rb] = 0;
        int64_t qoff;
        if constexpr (MODE == kCascade) {
            if (valid[rb]) hi[rb] = it.k_end;
            const int32_t e = valid[rb] ? it.row0 + r : it.row0;
            qoff = ((int64_t)a.rows[2 * e] * a.hq + a.rows[2 * e + 1]) * D;
        } else {
            const int qr = query_of(p0 + r);
            if (valid[rb]) row_interval(a, si, it, it.row0 + qr, lo[rb], hi[rb]);
            qoff = ((int64_t)(si.q_start + it.row0 + qr) * a.hq + head0 + (p0 + r - qr * g)) * D;
        }
#pragma unroll
        for (int s = 0; s < DS; ++s) {
            if (valid[rb]) {
                uint4 u = load16_nt(a.q, qoff + 32 * s + 8 * grp);
                qf[rb][s] = __builtin_bit_cast(bf16x8, u);
            } else {
                qf[rb][s] = bf16x8{};
            }
        }
    }
    if (grp == 0 && kg == 0) {
#pragma unroll
        for (int rb = 0; rb < RBW; ++rb) row_lohi[wave][rb * 16 + n] = make_int2(lo[rb], hi[rb]);
    }
    // wave-uniform bounds: intervals never shrink from one row to the next
    const int wr0 = wave * 16 * RBW;
    const int wr1 = min(wr0 + 16 * RBW - 1, np - 1);
    const bool wave_active = wr0 < np;
    int32_t w_lo_min = 0, w_lo_max = 0, w_hi_min = 0, w_hi_max = 0;
    if (wave_active) {
        if constexpr (MODE == kCascade) {
            w_hi_min = w_hi_max = it.k_end;  // lo = 0 for every row
        } else {
            row_interval(a, si, it, it.row0 + query_of(p0 + wr0), w_lo_min, w_hi_min);
            row_interval(a, si, it, it.row0 + query_of(p0 + wr1), w_lo_max, w_hi_max);
        }
    }
    // Keys of this workgroup's rows.  k_begin needs no row bounds (the window
    // alone moves it), so that the page indices can be requested beside them;
    // the loads themselves may run up to the item's end.
    int32_t k_end = it.k_end;
    int32_t k_begin = it.k_begin, rows_end = it.k_end;
    if (MODE == kPacked && g > 1) {
        const int32_t first = it.row0 + query_of(p0), last = it.row0 + query_of(p0 + np - 1);
        if (si.window > 0) k_begin = max(k_begin, (si.kv_len - si.q_len + first - si.window + 1) & ~(kPage - 1));
        k_begin = __builtin_amdgcn_readfirstlane(k_begin);
        rows_end = __builtin_amdgcn_readfirstlane(min(it.k_end, a.row_hi[si.hi_off + last]));
    }
    // Workgroups with more keys first, also within a CU: of those that share its
    // SIMDs the one with the most ends the launch, so its waves issue first, by
    // quarters of the launch's longest (four causal prompts of up to 1677 keys:
    // 60.4 -> 57.4 us, of 2000-8000 679 -> 671 against steps of 512 keys; one of
    // 12000 319 -> 321; equal items are unchanged) but at least 512 keys: with
    // lower steps 67 short rollouts, 275 and 422 keys at D = 64, take 104.9 us for
    // 102.4.  With key groups a CU has one workgroup, whose groups wait for each
    // other.
    if constexpr (KS == 1) {
        const int32_t span = rows_end - k_begin;
        if (span > 3 * a.span_step) __builtin_amdgcn_s_setprio(3);
        else if (span > 2 * a.span_step) __builtin_amdgcn_s_setprio(2);
        else if (span > a.span_step) __builtin_amdgcn_s_setprio(1);
    }
    // each key group takes an equal run of tiles (the last ones may be empty)
    const int total_tiles = (rows_end - k_begin + BN - 1) / BN;
    const int steps = KS == 1 ? total_tiles : (total_tiles + KS - 1) / KS;  // barriers of every wave
    const int n_tiles = KS == 1 ? total_tiles : min(steps, total_tiles - kg * steps);
    if constexpr (KS > 1) {
        k_begin += kg * steps * BN;
        k_end = min(k_end, k_begin + steps * BN);
    }

    float m[RBW], l[RBW];
    f32x4 o[RBW][DB];
#pragma unroll
    for (int rb = 0; rb < RBW; ++rb)
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] = f32x4{0, 0, 0, 0};
    // Rows past the item's end (never stored) start with reference 0, so that
    // the fixed mode below never meets an infinite reference.
#pragma unroll
    for (int rb = 0; rb < RBW; ++rb) {
        m[rb] = valid[rb] ? kNegInf : 0.0f;
        l[rb] = 0.0f;
    }

    // ---- LDS read offsets (per lane, the same for every tile) ----------------
    // K fragment (kb, s): row kb*16 + n, logical chunk 4 s + grp.
    uint32_t koff[DS];
    {
        const int sw = k_swizzle<D>(n);
#pragma unroll
        for (int s = 0; s < DS; ++s) koff[s] = n * RBY + (((4 * s + grp) ^ sw) << 4);
    }
    // V^T fragment (c, db, half h): row 32 c + 16 h + 4 grp + n / 4, bf16
    // column 16 db + 4 (n & 3), i.e. logical chunk 2 db + (n & 3) / 2.
    uint32_t voff[DB];
    {
        const int vr = 4 * grp + (n >> 2);
        const int vh = v_swizzle<D>(vr) >> 1;
        const uint32_t base = vr * RBY + (((n & 3) >> 1) << 4) + ((n & 1) << 3);
#pragma unroll
        for (int db = 0; db < DB; ++db) voff[db] = base + ((db ^ vh) << 5);
    }

    // ---- direct K/V loads ---------------------------------------------------
    // The item's page indices pass through a two-window LDS ring (64 pages =
    // 16 tiles per window).  Wave 0 fills a window with one direct-to-LDS dword
    // load (lane i writes page 64 w + i at ring[w & 1][i]) a whole window ahead
    // of its use; like the K/V loads it is covered by the wait at the top of
    // every tile.  Keeping the page indices out of compiler-tracked registers
    // matters: a tracked load in the loop makes the compiler wait for every
    // outstanding load (the just-issued K/V prefetch included) before its
    // result is first moved.  Load j of wave w fills rows (NW j + w) RPL ..
    // +RPL of the tile, which lie in one page; a thread's slot inside that
    // page and its logical chunk are the same for every tile and every j.
    const int32_t page0 = k_begin >> 4;
    const int32_t n_pages = ((k_end + 15) >> 4) - page0;
    const int32_t* bt_item = bt_row + page0;
    // window w of the item's pages: zeros past the last page (range check)
    auto load_window = [&](int w) {
        if (wave == 0 && 64 * w < n_pages) {
            // the pointer and size are wave-uniform; readfirstlane puts them in
            // scalar registers, where a buffer resource must live
            const uint64_t base = reinterpret_cast<uint64_t>(bt_item);
            const uint32_t lo32 = __builtin_amdgcn_readfirstlane((uint32_t)base);
            const uint32_t hi32 = __builtin_amdgcn_readfirstlane((uint32_t)(base >> 32));
            const __amdgpu_buffer_rsrc_t r =
                page_rsrc(reinterpret_cast<const char*>(((uint64_t)hi32 << 32) | lo32), 0,
                          (uint32_t)__builtin_amdgcn_readfirstlane(n_pages * 4));
            lds_dma4(r, (uint32_t)(64 * w + lane) * 4u, lds_address(&page_ring[w & 1][0]));
        }
    };
    bool page_err = false;
    const int64_t slot_stride = (int64_t)a.hkv * D;
    const uint32_t page_bytes = (uint32_t)(16 * slot_stride * sizeof(bf16_t));
    const int lrow0 = wave * RPL + lane / CH;  // tile row of load j = 0
    const int pch = lane % CH;                 // physical chunk this lane fills
    const uint32_t slot_off = (uint32_t)(((lrow0 & 15) * slot_stride + (int64_t)kvh * D) * sizeof(bf16_t));
    const uint32_t gk = slot_off + ((pch ^ k_swizzle<D>(lrow0)) << 4);
    const uint32_t gv = slot_off + ((pch ^ v_swizzle<D>(lrow0)) << 4);
    const char* kbase = reinterpret_cast<const char*>(a.k);
    const char* vbase = reinterpret_cast<const char*>(a.v);
    const __amdgpu_buffer_rsrc_t kpool = page_rsrc(kbase, 0, kSmallPoolBytes);
    const __amdgpu_buffer_rsrc_t vpool = page_rsrc(vbase, 0, kSmallPoolBytes);
    // Rows past the item's end read zeros through the buffer range check (their
    // offset is pushed out of range), and so does every row of a page outside
    // the pool: no access outside the pool, and zeros in LDS.
    constexpr uint32_t kOutOfRange = 0x80000000u;
    // LDS addresses of the two tile buffers (K at +0, V at +TB)
    const uint32_t lds_buf0 = __builtin_amdgcn_readfirstlane(lds_address(&buf0[0][0]));
    const uint32_t lds_buf1 = __builtin_amdgcn_readfirstlane(lds_address(&buf1[0][0]));
    // Page indices of tile tix for this wave's loads, read from the ring.
    // Load j of wave w fills tile rows (NW j + w) RPL .. +RPL, which lie in
    // page (NW j + w) RPL / 16 of the tile.  With four waves and RPL = 4
    // (d = 128) that page is j for every wave: one 8- or 16-byte LDS read
    // holds them.  Otherwise each wave reads its own indices at a
    // wave-uniform LDS address, with no per-lane selection.
    auto read_pages = [&](int tix, int32_t (&pv)[NLD]) {
        const int rel0 = tix * PPT;
        const int32_t* ring = &page_ring[(rel0 >> 6) & 1][rel0 & 63];
        if constexpr (NW == 4 && RPL == 4 && NLD == 4) {
            const int4 pq = *reinterpret_cast<const int4*>(ring);
            pv[0] = pq.x; pv[1] = pq.y; pv[2] = pq.z; pv[3] = pq.w;
        } else if constexpr (NW == 4 && RPL == 4 && NLD == 2) {
            const int2 pq = *reinterpret_cast<const int2*>(ring);
            pv[0] = pq.x; pv[1] = pq.y;
        } else {
#pragma unroll
            for (int j = 0; j < NLD; ++j) pv[j] = ring[((NW * j + wave) * RPL) >> 4];
        }
    };
    // Loads of tile tix into the buffer at LDS address `dst` ([K, V]), with
    // the page indices `pv` read one tile earlier (so that the LDS round trip
    // of the read overlaps a tile's compute); then the indices of tile tix + 1.
    int32_t pv[NLD];
    auto issue_tile = [&](int tix, uint32_t dst) {
        const int rel0 = tix * PPT;
        uint32_t page[NLD];
#pragma unroll
        for (int j = 0; j < NLD; ++j) page[j] = (uint32_t)__builtin_amdgcn_readfirstlane(pv[j]);
        // first tile of window w >= 1: every wave is past its last read of
        // window w - 1, so its ring slot can take window w + 1 (tile tix + 1
        // lies in window w, or in w + 1 only if tix ends window w, whose
        // successor has landed long before)
        if (tix > 0 && (rel0 & 63) == 0) load_window((rel0 >> 6) + 1);
        if (tix + 1 < n_tiles) read_pages(tix + 1, pv);
        bool all_ok = true;
#pragma unroll
        for (int j = 0; j < NLD; ++j) all_ok &= page[j] < (uint32_t)a.num_pages;
        const int32_t k0 = k_begin + tix * BN;
        const bool tail = k0 + BN > k_end;
        if (__builtin_expect(SMALL && all_ok && !tail, 1)) {
            // common case: only the page offsets change from tile to tile
#pragma unroll
            for (int j = 0; j < NLD; ++j) {
                const uint32_t soff = page[j] * page_bytes;
                lds_dma16s(kpool, gk, soff, dst + (NW * j + wave) * 1024);
                lds_dma16s(vpool, gv, soff, dst + TB + (NW * j + wave) * 1024);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NLD; ++j) {
                const int pg = ((NW * j + wave) * RPL) >> 4;  // page of this load within the tile
                const bool ok = page[j] < (uint32_t)a.num_pages;
                page_err |= !ok && k0 + 16 * pg < k_end;
                const bool live = ok && (!tail || k0 + lrow0 + NW * j * RPL < k_end);
                if (SMALL) {
                    const uint32_t soff = ok ? page[j] * page_bytes : 0u;
                    lds_dma16s(kpool, live ? gk : kOutOfRange, soff, dst + (NW * j + wave) * 1024);
                    lds_dma16s(vpool, live ? gv : kOutOfRange, soff, dst + TB + (NW * j + wave) * 1024);
                } else {
                    const size_t pofs = ok ? (size_t)page[j] * page_bytes : 0;
                    const uint32_t nrec = ok ? page_bytes : 0u;
                    lds_dma16s(page_rsrc(kbase, pofs, nrec), live ? gk : kOutOfRange, 0u,
                               dst + (NW * j + wave) * 1024);
                    lds_dma16s(page_rsrc(vbase, pofs, nrec), live ? gv : kOutOfRange, 0u,
                               dst + TB + (NW * j + wave) * 1024);
                }
            }
        }
    };

    // ---- 4-bit loads and conversion ------------------------------------------
    // wave w's share of a tile: page w % PPT of it, K for the first PPT waves and
    // V for the others (two pages), or both (four)
    typedef Record<D> R;
    constexpr bool BOTH = PPT == NW;
    const int share_page = wave % PPT;
    const bool share_v = wave >= PPT;
    constexpr int NC4 = D / 32;  // dwords of codes per lane and record
    struct Raw {
        uint32_t code[BOTH ? 2 * NC4 : NC4];  // with both: K, then V
        uint32_t scale, vs;                   // with both: of K (one byte) and of V
    } raw;
    auto load_codes = [&](__amdgpu_buffer_rsrc_t r, uint32_t* x) {
        if constexpr (D == 128) {
            const uint4 c = load16_at(r, lane * 16);
            x[0] = c.x; x[1] = c.y; x[2] = c.z; x[3] = c.w;
        } else {
            typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
            const u32x2 c = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(r, lane * 8, 0, 0));
            x[0] = c[0]; x[1] = c[1];
        }
    };
    // The item's page indices pass through two registers of 64 (a lane each): a
    // scalar load in the tile loop would make every wait for LDS reads a wait for
    // all of them.  Pages past the last one are -1, and no load sits in a branch,
    // where it could not be counted.
    auto page_window = [&](int w) { return 64 * w + lane < n_pages ? bt_item[64 * w + lane] : -1; };
    int32_t pw_cur = -1, pw_next = -1;
    auto load4 = [&](int tix) {
        const int rel = tix * PPT;
        if (rel > 0 && (rel & 63) == 0) {
            pw_cur = pw_next;
            pw_next = page_window((rel >> 6) + 1);
        }
        const int32_t page = __builtin_amdgcn_readlane(pw_cur, (rel & 63) + share_page);
        const bool ok = (uint32_t)page < (uint32_t)a.num_pages;
        page_err |= !ok && rel + share_page < n_pages;
        const size_t ofs = ok ? ((size_t)page * a.hkv + kvh) * R::kBytes : 0;
        const uint32_t nrec = ok ? (uint32_t)R::kBytes : 0u;  // else reads zeros
        // four scale bytes of V; of K the one byte (with both), or those of keys n & ~3 .. n | 3
        const uint32_t kscale = R::kScales + (grp * (D / 4) / 32) * 16 + (BOTH ? n : n & ~3);
        const uint32_t vscale = R::scale(4 * grp, n);
        if constexpr (BOTH) {
            const __amdgpu_buffer_rsrc_t rk = page_rsrc(kbase, ofs, nrec), rv = page_rsrc(vbase, ofs, nrec);
            load_codes(rk, raw.code);
            load_codes(rv, raw.code + NC4);
            raw.scale = __builtin_amdgcn_raw_buffer_load_b8(rk, (int)kscale, 0, 0);
            raw.vs = __builtin_amdgcn_raw_buffer_load_b32(rv, (int)vscale, 0, 0);
        } else {
            const __amdgpu_buffer_rsrc_t r = page_rsrc(share_v ? vbase : kbase, ofs, nrec);
            load_codes(r, raw.code);
            raw.scale = __builtin_amdgcn_raw_buffer_load_b32(r, (int)(share_v ? vscale : kscale), 0, 0);
        }
    };
    // Where the lane's converted pieces go: the rows and swizzles differ in bits of
    // their own, so that piece i is at one base with a few bits flipped.
    //  K: row n of the page, 16-byte chunks D / 32 grp + i;
    //  V: rows 4 grp + i, D / 16 dims from n D / 16 on.
    const int k_row = share_page * 16 + n, v_row = share_page * 16 + 4 * grp;
    const uint32_t k_at = k_row * RBY + (((grp * (D / 32)) ^ k_swizzle<D>(k_row)) << 4);
    const uint32_t v_at = TB + v_row * RBY + (((n * D / 128) ^ v_swizzle<D>(v_row)) << 4) + (D == 64 ? (n & 1) * 8 : 0);
    auto v_flip = [](int i) { return D == 128 ? i * 0x120 : i * 0x80 + (i >> 1) * 0x20; };
    const uint32_t at4 = share_v ? v_at : k_at, flip4 = share_v ? 0x120 : 0x10;
    // picks the scale of each piece: V's four as they are, K's one for all
    const uint32_t k_pick = (n & 3) * 0x01010101u, pick4 = share_v ? 0x03020100u : k_pick;
    auto store4 = [&](char (&dst)[2][TB]) {
        char* to = &dst[0][0];
        if constexpr (BOTH) {
            const float sk = scale_of(raw.scale);
#pragma unroll
            for (int i = 0; i < NC4; ++i)
                *reinterpret_cast<bf16x8*>(to + (k_at ^ (i * 0x10))) = eight_of(raw.code[i], sk);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float sv = scale_of(v_scale(raw.vs, i));
                if constexpr (D == 128) {
                    *reinterpret_cast<bf16x8*>(to + (v_at ^ v_flip(i))) = eight_of(raw.code[NC4 + i], sv);
                } else {
                    const uint32_t w = raw.code[NC4 + (i >> 1)];
                    *reinterpret_cast<bf16x4*>(to + (v_at ^ v_flip(i))) = (i & 1) ? four_of<2>(w, sv) : four_of<0>(w, sv);
                }
            }
        } else {
            const uint32_t* w = raw.code;
            const uint32_t sc = __builtin_amdgcn_perm(raw.scale, raw.scale, pick4);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<bf16x8*>(to + (at4 ^ (i * flip4))) = eight_of(w[i], scale_of(v_scale(sc, i)));
        }
    };

    // ---- one tile: scores, mask, online softmax, weighted values ---------------
    const float c2 = a.scale_log2;
    auto scores = [&](const char* kl, f32x4 (&sc)[RBW][NB]) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) {
            bf16x8 kf[DS];
#pragma unroll
            for (int s = 0; s < DS; ++s) kf[s] = *reinterpret_cast<const bf16x8*>(kl + kb * 16 * RBY + koff[s]);
#pragma unroll
            for (int rb = 0; rb < RBW; ++rb) sc[rb][kb] = mfma16(kf[0], qf[rb][0], f32x4{0, 0, 0, 0});
#pragma unroll
            for (int s = 1; s < DS; ++s)
#pragma unroll
                for (int rb = 0; rb < RBW; ++rb) sc[rb][kb] = mfma16(kf[s], qf[rb][s], sc[rb][kb]);
        }
    };
    auto mask = [&](int32_t k0, f32x4 (&sc)[RBW][NB]) {
#pragma unroll
        for (int rb = 0; rb < RBW; ++rb) {
            // key k0 + 4 grp + c is visible iff lo <= key < hi
            const int2 lh = row_lohi[wave][rb * 16 + n];
            const int32_t lo_r = lh.x - (k0 + 4 * grp), hi_r = lh.y - (k0 + 4 * grp);
#pragma unroll
            for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = kb * 16 + i;
                    if (!(c >= lo_r && c < hi_r)) sc[rb][kb][i] = kNegInf;
                }
        }
    };
    // probabilities as the bf16 B operands of the value product (32-key halves)
    auto pack = [&](const f32x4 (&sc)[RBW][NB], bf16x8 (&pf)[NC][RBW]) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
            for (int rb = 0; rb < RBW; ++rb) pf[c][rb] = to_bf16x8(sc[rb][2 * c], sc[rb][2 * c + 1]);
    };
    auto values = [&](const char* vl, const bf16x8 (&pf)[NC][RBW]) {
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            bf16x8 vf[DB];
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16_t* base = reinterpret_cast<const bf16_t*>(vl + 32 * c * RBY + voff[db]);
                vf[db] = cat(lds_read_tr16(base), lds_read_tr16(base + 16 * D));
            }
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int rb = 0; rb < RBW; ++rb) o[rb][db] = mfma16(vf[db], pf[c][rb], o[rb][db]);
        }
    };
    // Two softmax modes.  Exact: the tile's row maxima are taken and the
    // reference moved lazily (softmax_update); used on a wave's tiles until
    // every valid row of the wave has a reference.  Fixed: probabilities
    // against each row's reference as it stands, with no maximum at all (an
    // fma, an exp2 and a sum per score), which takes the reductions and the
    // cross-lane exchange out of the tile.  Both are exact (out = O / l and
    // lse = m + log2 l share the reference).  A fixed-mode tile whose sums
    // reach kFixedTileLimit (scores far above the reference) is redone in exact
    // mode from its scores, recomputed from the K tile still in LDS.
    bool need_ref = true;  // wave-uniform: some valid row of the wave has no reference yet
    auto exact_update = [&](f32x4 (&sc)[RBW][NB]) {
        float alpha[RBW];
        if (softmax_update<RBW, NB>(rg, sc, c2, m, l, alpha)) {
#pragma unroll
            for (int rb = 0; rb < RBW; ++rb)
#pragma unroll
                for (int db = 0; db < DB; ++db) o[rb][db] *= alpha[rb];
        }
    };
    auto compute_tile = [&](int tix, const char (&cur)[2][TB]) {
        const int32_t k0 = k_begin + tix * BN;
        if (!(wave_active && k0 < w_hi_max && k0 + BN > w_lo_min)) return;
        // the compiler's interleaving strategy for LDS reads among MFMAs
        // (1-2% at d = 128, neutral at d = 64)
        __builtin_amdgcn_iglp_opt(0);
        const char* kl = &cur[0][0];
        const char* vl = &cur[1][0];
        const bool full = k0 >= w_lo_max && k0 + BN <= w_hi_min;
        f32x4 sc[RBW][NB];
        bf16x8 pf[NC][RBW];
        scores(kl, sc);
        if (!full) mask(k0, sc);
        bool exact = need_ref;
        if (!need_ref) {
            float ts[RBW];
            softmax_fixed<RBW, NB>(sc, c2, m, ts);
            bool over = false;
#pragma unroll
            for (int rb = 0; rb < RBW; ++rb) over |= !(ts[rb] < kFixedTileLimit);
            exact = __builtin_amdgcn_ballot_w64(over) != 0;
            if (!exact) {
#pragma unroll
                for (int rb = 0; rb < RBW; ++rb) l[rb] += ts[rb];
                pack(sc, pf);
            }
        }
        if (exact) {
            if (!need_ref) {
                // a fixed-mode tile out of range: its scores again, from an
                // opaque copy of the K tile's address so that the compiler
                // loads the fragments anew instead of keeping the first ones
                // (and the raw scores) alive through the softmax
                uint32_t ka = lds_address(kl);
                asm volatile("" : "+s"(ka));
                scores((const char*)((const lds_char*)(uintptr_t)ka), sc);
                if (!full) mask(k0, sc);
            }
            exact_update(sc);
            bool missing = false;
#pragma unroll
            for (int rb = 0; rb < RBW; ++rb) missing |= m[rb] == kNegInf;
            need_ref = __builtin_amdgcn_ballot_w64(missing) != 0;
            pack(sc, pf);
        }
        values(vl, pf);
    };

    if (CACHE != kPool4 && steps > 0) {
        load_window(0);
        load_window(1);
        // The Q fragments are consumed here, so the compiler's wait for their
        // loads sits before any K/V load is in flight.
#pragma unroll
        for (int rb = 0; rb < RBW; ++rb)
#pragma unroll
            for (int s = 0; s < DS; ++s) asm volatile("" ::"v"(qf[rb][s]));
        dma_barrier();  // windows 0 and 1 of the page ring have landed
        if (KS == 1 || n_tiles > 0) {
            read_pages(0, pv);
            issue_tile(0, lds_buf0);
        }
        // Tile tix is in buf[tix & 1].  At the top of each tile every wave has
        // its own loads of the tile done (vmcnt) and every wave is done with
        // the other buffer (barrier), which the next tile's loads then take.
        for (int tix = 0; tix < steps; tix += 2) {
            dma_barrier();
            if (tix + 1 < n_tiles) issue_tile(tix + 1, lds_buf1);
            if (KS == 1 || tix < n_tiles) compute_tile(tix, buf0);
            if (tix + 1 < steps) {
                dma_barrier();
                if (tix + 2 < n_tiles) issue_tile(tix + 2, lds_buf0);
                if (KS == 1 || tix + 1 < n_tiles) compute_tile(tix + 1, buf1);
            }
        }
    }
    if constexpr (CACHE == kPool4) {
        // As above, but tile t + 1 goes from registers into the other buffer at
        // the top of tile t, and the loads of tile t + 2 follow it.
        pw_cur = page_window(0);
        pw_next = page_window(1);
        load4(0);
        store4(buf0);
        load4(1);
        auto top = [&](int tix, char (&next)[2][TB]) {
            lds_barrier();
            store4(next);
            load4(tix + 2);
        };
        for (int tix = 0; tix < steps; tix += 2) {
            top(tix, buf1);
            if (KS == 1 || tix < n_tiles) compute_tile(tix, buf0);
            if (tix + 1 < steps) {
                top(tix + 1, buf0);
                if (KS == 1 || tix + 1 < n_tiles) compute_tile(tix + 1, buf1);
            }
        }
    }
    if (page_err && lane == 0) atomicOr(a.err, MSTAR_DEVERR_PAGE_RANGE_BIT);

    // ---- epilogue -------------------------------------------------------------
    float lt[RBW];
#pragma unroll
    for (int rb = 0; rb < RBW; ++rb) lt[rb] = rg.sum(l[rb]);
    if constexpr (KS > 1) {
        // the key groups' results against the largest reference, summed into
        // group 0 through LDS (the tile buffers are done with)
        constexpr int R = 64 * RBW;  // rows
        static_assert(R * D * 4 <= (int)sizeof(bufs), "one group's O^T fits in the tile buffers");
        float* ml = reinterpret_cast<float*>(&bufs[0][0][0][0]);
        dma_barrier();
#pragma unroll
        for (int rb = 0; rb < RBW; ++rb)
            if (grp == 0) {
                ml[(2 * kg) * R + (wave * RBW + rb) * 16 + n] = m[rb];
                ml[(2 * kg + 1) * R + (wave * RBW + rb) * 16 + n] = lt[rb];
            }
        dma_barrier();
#pragma unroll
        for (int rb = 0; rb < RBW; ++rb) {
            const int row = (wave * RBW + rb) * 16 + n;
            float mstar = kNegInf, L = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) mstar = fmax_num(mstar, ml[2 * k * R + row]);
            const float mu = mstar == kNegInf ? 0.0f : mstar;
#pragma unroll
            for (int k = 0; k < KS; ++k) L += fast_exp2(ml[2 * k * R + row] - mu) * ml[(2 * k + 1) * R + row];
            const float own = fast_exp2(m[rb] - mu);
#pragma unroll
            for (int db = 0; db < DB; ++db) o[rb][db] *= own;
            m[rb] = mstar;
            lt[rb] = L;
        }
        f32x4* sum = reinterpret_cast<f32x4*>(&bufs[0][0][0][0]);  // [16-byte piece][thread of the group]
#pragma unroll
        for (int k = 1; k < KS; ++k) {
            dma_barrier();
            if (kg == k) {
#pragma unroll
                for (int rb = 0; rb < RBW; ++rb)
#pragma unroll
                    for (int db = 0; db < DB; ++db) sum[(rb * DB + db) * 256 + wave * 64 + lane] = o[rb][db];
            }
            dma_barrier();
            if (kg == 0) {
#pragma unroll
                for (int rb = 0; rb < RBW; ++rb)
#pragma unroll
                    for (int db = 0; db < DB; ++db) o[rb][db] += sum[(rb * DB + db) * 256 + wave * 64 + lane];
            }
        }
        if (kg != 0) return;
    }
    int pe = p0;  // opaque: the rows' divisions are done again rather than kept through the tile loop
    asm volatile("" : "+s"(pe));
#pragma unroll
    for (int rb = 0; rb < RBW; ++rb) {
        if (!valid[rb]) continue;
        const int r = wave * 16 * RBW + rb * 16 + n;
        const float inv = lt[rb] > 0.0f ? 1.0f / lt[rb] : 0.0f;
        const float lse = lt[rb] > 0.0f ? (m[rb] + __log2f(lt[rb])) * kLn2 : kNegInf;
        if constexpr (MODE == kCascade) {
            const int64_t slot = it.part + r;  // cascade items always write partials
            float* po = a.part_o + slot * D;
#pragma unroll
            for (int db = 0; db < DB; ++db)
                *reinterpret_cast<f32x4*>(po + db * 16 + 4 * grp) = o[rb][db] * inv;
            if (grp == 0) a.part_lse[slot] = lse;
        } else if (it.part < 0) {
            const int qr = query_of(pe + r);
            const int64_t row = (int64_t)(si.q_start + it.row0 + qr) * a.hq + head0 + (pe + r - qr * g);
            bf16_t* out = reinterpret_cast<bf16_t*>(a.out) + row * D;
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const bf16x4 v = __builtin_convertvector(o[rb][db] * inv, bf16x4);
                *reinterpret_cast<bf16x4*>(out + db * 16 + 4 * grp) = v;
            }
            if (grp == 0) a.lse[row] = lse;
        } else {
            const int qr = query_of(pe + r);
            const int64_t slot = it.part + (int64_t)(head0 + (pe + r - qr * g)) * it.head_stride + qr;
            float* po = a.part_o + slot * D;
#pragma unroll
            for (int db = 0; db < DB; ++db)
                *reinterpret_cast<f32x4*>(po + db * 16 + 4 * grp) = o[rb][db] * inv;
            if (grp == 0) a.part_lse[slot] = lse;
        }
    }
}

}  // namespace
}  // namespace mstar
