// HIP kernels of the operators on paged caches (mstar_cache.h) for gfx950: the
// 4-bit cache's append, attention and read-back, and block tables.
#include <algorithm>

#include "tile.h"

namespace mstar {
namespace {

// ---------------------------------------------------------------------------
// Append: a workgroup takes up to 16 new rows of one request, a wave one KV head
// of them at a time, by aligned groups of four positions (at most five): lane
// 4 n + j holds dims [n D / 16, +D / 16) of a group's key j, so that its V words
// are consecutive and its K words run over 64 (D = 128) or 32 bytes of each
// piece.  The 32 dims of a scale are 4 (D = 128) or 8 neighbouring n.
//
// Bound: HBM and the chain of reads before it (item, request, rows and page
// indices).  34816 rows of 4 heads at D = 128 (71 MB read, 19 MB written) take 24
// us, 3.7 TB/s; with element-wise loads behind the page indices, and each code found
// by comparisons, it was 40.
// ---------------------------------------------------------------------------
// A lane's D / 16 bf16 values as packed pairs.
template <int D>
struct Piece {
    uint32_t w[D / 32];
};
template <int D>
__device__ __forceinline__ Piece<D> load_piece(const void* rows, int64_t elem) {
    Piece<D> p;
    if constexpr (D == 128) {
        const uint4 u = load16_nt(rows, elem);
        p.w[0] = u.x; p.w[1] = u.y; p.w[2] = u.z; p.w[3] = u.w;
    } else {
        typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
        const u32x2 u = __builtin_nontemporal_load(reinterpret_cast<const u32x2*>(static_cast<const bf16_t*>(rows) + elem));
        p.w[0] = u[0]; p.w[1] = u[1];
    }
    return p;
}

// Codes (one byte per pair) and scale byte of a lane's piece, whose block's other
// dims are with the lanes that differ in bits 2, 3 (and 4 at D = 64).  The scale
// is exact; the conversion divides by it and rounds once, to the nearest code,
// ties to even.  `odd` tells of an infinity or a NaN; NaN becomes 0.
template <int D>
__device__ __forceinline__ uint32_t round_piece(Piece<D>& p, int& b, bool& odd) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top2 = {0, 0};
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
        top2 = __builtin_elementwise_max(top2, __builtin_bit_cast(u16x2, p.w[i] & 0x7fff7fffu));
    uint32_t top = max((uint32_t)top2[0], (uint32_t)top2[1]);
    if (top >= 0x7f80u) {
        odd = true;
        top = 0;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            uint32_t lo = p.w[i] & 0xffffu, hi = p.w[i] >> 16;
            if ((lo & 0x7fffu) > 0x7f80u) lo = 0;
            if ((hi & 0x7fffu) > 0x7f80u) hi = 0;
            p.w[i] = lo | (hi << 16);
            top = max(top, max(lo & 0x7fffu, hi & 0x7fffu));
        }
    }
    top = max(top, (uint32_t)__shfl_xor((int)top, 4, 64));
    top = max(top, (uint32_t)__shfl_xor((int)top, 8, 64));
    if (D == 64) top = max(top, (uint32_t)__shfl_xor((int)top, 16, 64));
    // smallest b with top <= 7 * 2^(b - 127): 7 is mantissa 0x60 two binades up
    b = min(max((int)((top + 31) >> 7) - 2, kScaleMin), kScaleMax);
    const float s = scale_of((uint32_t)b);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, p.w[0]), s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, p.w[1]), s, 1);
    if constexpr (D == 128) {
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, p.w[2]), s, 2);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, p.w[3]), s, 3);
    }
    return c;
}

template <int D>
__global__ __launch_bounds__(256) void append4_kernel(Append4Args a) {
    constexpr int E = D / 16;        // dims per lane
    constexpr int GR = kAppendRows / 4 + 1;  // groups of four positions that 16 rows touch
    typedef Record<D> R;
    const WorkItem it = a.items[wg_id()];
    const SeqInfo si = a.seqs[it.seq];
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3, lane = thread_id() & 63;
    const int n = lane >> 2, j = lane & 3;
    const int32_t* bt_row = a.bt + (int64_t)it.seq * a.bt_stride;
    const int32_t p0 = it.k_begin & ~3;
    bool live[GR], bad_page = false, bad_value = false;
    int32_t page[GR];
#pragma unroll
    for (int g = 0; g < GR; ++g) {
        const int32_t pos = p0 + 4 * g + j;
        live[g] = pos >= it.k_begin && pos < it.k_end;
        page[g] = live[g] ? bt_row[pos >> 4] : 0;
    }
    const int64_t row0 = si.q_start + (p0 + j - (si.kv_len - si.q_len));
    for (int head = wave; head < a.hkv; head += 4) {
        // every row's loads before any is used, and before the page indices are
        Piece<D> k[GR], v[GR];
#pragma unroll
        for (int g = 0; g < GR; ++g) {
            k[g] = v[g] = Piece<D>{};
            if (live[g]) {
                const int64_t src = ((row0 + 4 * g) * a.hkv + head) * D + n * E;
                k[g] = load_piece<D>(a.k_new, src);
                v[g] = load_piece<D>(a.v_new, src);
            }
        }
#pragma unroll
        for (int g = 0; g < GR; ++g) {
            if (p0 + 4 * g >= it.k_end) continue;
            int kb, vb;
            const uint32_t kw = round_piece<D>(k[g], kb, bad_value), vw = round_piece<D>(v[g], vb, bad_value);
            if (!live[g]) continue;
            if ((uint32_t)page[g] >= (uint32_t)a.num_pages) {
                bad_page = true;
                continue;
            }
            const int slot = (p0 + 4 * g + j) & 15;
            const int64_t rec = ((int64_t)page[g] * a.hkv + head) * R::kBytes;
            char* kr = static_cast<char*>(a.k) + rec;
            char* vr = static_cast<char*>(a.v) + rec;
            if constexpr (D == 128) {
                *reinterpret_cast<uint32_t*>(kr + R::k_word(slot, n)) = kw;
                *reinterpret_cast<uint32_t*>(vr + R::v_word(slot, n)) = vw;
            } else {
                *reinterpret_cast<uint16_t*>(kr + R::k_word(slot, n)) = (uint16_t)kw;
                *reinterpret_cast<uint16_t*>(vr + R::v_word(slot, n)) = (uint16_t)vw;
            }
            if (n % (32 / E) == 0) {
                kr[R::scale(slot, n)] = (char)kb;
                vr[R::scale(slot, n)] = (char)vb;
            }
        }
    }
    const int bits = (__builtin_amdgcn_ballot_w64(bad_page) ? MSTAR_DEVERR_PAGE_RANGE_BIT : 0) |
                     (__builtin_amdgcn_ballot_w64(bad_value) ? MSTAR_DEVERR_NONFINITE_BIT : 0);
    if (bits && lane == 0) atomicOr(a.err, bits);
}

// ---------------------------------------------------------------------------
// Unpack: a wave takes one record of a listed page, four keys at a time; lane
// 16 g + n writes dims [n D / 16, +D / 16) of the group's key g.
//
// Bound: HBM, mostly the pages written.  Rows that the append reads and pages that
// this writes are non-temporal: 34816 rows of 4 heads stored and read back (D =
// 128, 180 MB) 48 -> 39 us, of which this kernel takes 15.4 (5.8 TB/s).
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void store_word(bf16_t* out, uint32_t w, float s) {
    typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
    typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
    if constexpr (D == 128)
        __builtin_nontemporal_store(__builtin_bit_cast(u32x4, eight_of(w, s)), reinterpret_cast<u32x4*>(out));
    else
        __builtin_nontemporal_store(__builtin_bit_cast(u32x2, four_of<0>(w, s)), reinterpret_cast<u32x2*>(out));
}

template <int D>
__global__ __launch_bounds__(256) void unpack4_kernel(Unpack4Args a) {
    typedef Record<D> R;
    const int wave = __builtin_amdgcn_readfirstlane(thread_id() >> 6) & 3, lane = thread_id() & 63;
    const int g = lane >> 4, n = lane & 15;
    const int64_t tasks = (int64_t)a.n_ids * a.hkv;
    for (int64_t task = (int64_t)wg_id() * 4 + wave; task < tasks; task += 4 * (int64_t)a.n_wgs) {
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
}

// ---------------------------------------------------------------------------
// Block tables: a thread per new row.  The row that starts a page enters it; rows
// of one page read the same entry of the free list, whose offset per request is in
// the plan, so no thread waits for another.
//
// Bound: the launch (4.1 us for 64 rows, 4.7 for 307200 and 2.5 MB of slots).
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
    // a wave per record, in several turns past 2^20 workgroups
    Unpack4Args b = a;
    b.n_wgs = (int32_t)std::min<int64_t>(((int64_t)a.n_ids * a.hkv + 3) / 4, 1 << 20);
    return launch(head_dim == 64 ? unpack4_kernel<64> : unpack4_kernel<128>, dim3(b.n_wgs), dim3(256), b, s);
}

namespace {
// Keys per tile at D = 128: 32, with three workgroups per CU, or 64 with two
// (half the barriers per key and twice the independent work per wave) where a
// launch leaves a CU no more than two anyway: two prompts of 1000 tokens, 28/4 heads
// (448 workgroups), 35.8 -> 33.3 us; one of 600 (168) 21.4 -> 20.5.  Past that either
// wins, the losses being larger: one of 1500, 28/4 (560), 45.3 -> 42.6, eight of 300
// (672) 24.4 -> 23.4, but 20 of 200, 16/8 (640), 21.1 -> 26.8.  With key groups two of 64 keys for three of 32:
// one prompt of 1000 tokens, 8/2 heads, 25.2 -> 24.4, 1500, 4/4, 29.3 -> 27.8; two of
// 1846, 8/2, 38.7 -> 39.0.  Three key groups at D = 64, where a fourth leaves the
// conversion too few registers: one prompt of 700 tokens, 16/8 heads, 17.6 -> 14.8,
// of 1500 28.0 -> 24.7.
constexpr int kTwoPerCu = 512;

template <int MODE, int BN128, int KS64, int KS128>
hipError_t launch_tile4_mode(const KArgs& a, int head_dim, hipStream_t s) {
    const dim3 g((unsigned)a.n_wgs);
    return head_dim == 64 ? launch(tile_kernel<64, 2, kPool4, MODE, 64, KS64>, g, dim3(256 * KS64), a, s)
                          : launch(tile_kernel<128, 2, kPool4, MODE, BN128, KS128>, g, dim3(256 * KS128), a, s);
}
template <int MODE>
hipError_t launch_tile4_rows(const KArgs& a, int head_dim, hipStream_t s) {
    if (a.key_groups) return launch_tile4_mode<MODE, 64, 3, 2>(a, head_dim, s);
    return a.n_wgs <= kTwoPerCu ? launch_tile4_mode<MODE, 64, 1, 1>(a, head_dim, s)
                                : launch_tile4_mode<MODE, 32, 1, 1>(a, head_dim, s);
}
}  // namespace

// As launch_tiles, launch_cascade and launch_few for a 16-bit cache.
hipError_t launch_tiles4(const KArgs& a, int head_dim, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    return a.group_inv != 0 ? launch_tile4_rows<kPacked>(a, head_dim, s) : launch_tile4_rows<kRows>(a, head_dim, s);
}

hipError_t launch_cascade4(const KArgs& a, int head_dim, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    return launch_tile4_mode<kCascade, 32, 1, 1>(a, head_dim, s);
}

namespace {
// At D = 128 few-row items take the tiles' LDS, so tiles of 64 keys also halve how many
// items a CU holds.  They are taken where few workgroups wait for that (three a CU,
// tiles and items together), us with 32 -> 64 keys: 4 decode steps beside three
// prompts of 400 tokens, 16/8 heads (192 tiles, 544 items), 24.9 -> 23.1; beside two of
// 600, 28/4 (280, 272), 30.2 -> 29.0; 40 behind a prefix of 16384, 28/4 (264, 296),
// 39.0 -> 36.3.  From there to 900 either wins (4 beside one of 1500, 16/8, 256 and 544,
// 45.5 -> 40.9; 32 beside two of 300, 28/4, 168 and 708, 23.5 -> 26.2), past it 32 keys
// (32 beside three of 400, 28/4, 392 and 708, 30.4 -> 32.9).
// Or where a cascade's longest item has at least as many keys as there are few-row
// items.  The item is a chain of its keys, which longer tiles shorten; the items' turns
// grow with their number and with the keys of each, which the rule does not see, so
// the ratio is a fit that errs to 32 keys.  Above it 64 won in each of seven cascades
// (128 behind 12288, 28/4, 1280 keys and 908 items, 61.9 -> 57.1; 200 behind 16384,
// 16/8, 2048 and 1600, 69.0 -> 61.9; 100 behind 32768, 8/8, 1024 and 800, 44.6 -> 41.8;
// 600 behind 4096, 8/1, 640 and 600, 37.8 -> 37.2).  Below it either wins: gains not
// taken are 128 behind 6144 and 8192, 28/4 (640 and 832, 908), 41.5 -> 39.0 and 47.8 ->
// 44.7, and 300 behind 3584 (896, 1200), 52.5 -> 47.7; losses spared 200 behind 8192,
// 16/8 (1024, 1600), 45.2 -> 50.4, behind 4096 (512, 1600) 38.4 -> 43.9, 100 behind
// 16384, 8/8 (512, 800), 33.1 -> 36.3, and 300 behind 2048, 28/4 (512, 1200), 40.2 ->
// 42.1.
constexpr int kThreePerCu = 768;

template <int MODE, int RB>
hipError_t launch_mixed4_mode(const MixedArgs& a, int head_dim, hipStream_t s) {
    const dim3 g((unsigned)a.tile.n_wgs + (unsigned)a.few.n_items), b(256);
    if (head_dim == 64) return launch(tile_kernel<64, 2, kPool4, MODE, 64, 1, RB>, g, b, a, s);
    const bool long_keys = a.tile.n_wgs <= kTwoPerCu &&
                           ((int64_t)a.tile.n_wgs + a.few.n_items <= kThreePerCu ||
                            (MODE == kCascade && a.tile.span >= a.few.n_items));
    return long_keys ? launch(tile_kernel<128, 2, kPool4, MODE, 64, 1, RB>, g, b, a, s)
                     : launch(tile_kernel<128, 2, kPool4, MODE, 32, 1, RB>, g, b, a, s);
}
template <int RB>
hipError_t launch_mixed4_rows(const MixedArgs& a, bool cascade, int head_dim, hipStream_t s) {
    if (cascade) return launch_mixed4_mode<kCascade, RB>(a, head_dim, s);
    return a.tile.group_inv != 0 ? launch_mixed4_mode<kPacked, RB>(a, head_dim, s)
                                 : launch_mixed4_mode<kRows, RB>(a, head_dim, s);
}
}  // namespace

hipError_t launch_mixed4(const KArgs& tile, const KArgs& few, bool cascade, int head_dim, int rb, hipStream_t s) {
    MixedArgs a{};
    a.tile = tile;
    a.few = few;
    a.done = tile.done;
    return rb == 1 ? launch_mixed4_rows<1>(a, cascade, head_dim, s) : launch_mixed4_rows<2>(a, cascade, head_dim, s);
}

namespace {
// Eight waves per item, for four, where the items leave a CU room for them (as many
// as its registers hold: two workgroups, or one of more rows).  us with four -> eight:
//   D = 64, 16/8 heads: 64 decode steps over 4000 keys (512 items)   39.0 -> 31.3
//                       64 12-token chunks over 2000 (512)           27.8 -> 24.3
//   D = 128, 28/4:      128 decode steps over 1500 (512)             22.6 -> 20.8
//                       one over 1500 (24)                            9.1 ->  8.8
//                       8 over 2000 (256)                             9.6 ->  9.6
//   D = 128, 16/8:      32 16-token chunks over 2000 (256)           25.7 -> 20.7
// Past that they lose, at D = 64 and 12/12 heads:
//                       50 decode steps over 3000 (600)              33.4 -> 35.1
//                       64 over 600 (768)                            10.6 -> 13.6
template <int D, int RB>
hipError_t launch_few4_rows(const KArgs& a, hipStream_t s) {
    constexpr int kPerCu = RB == 1 || (D == 64 && RB == 2) ? 2 : 1;
    const dim3 g(a.n_items);
    return a.n_items <= 256 * kPerCu ? launch(few4_kernel<D, RB, 8>, g, dim3(512), a, s)
                                     : launch(few4_kernel<D, RB, 4>, g, dim3(256), a, s);
}
}  // namespace

hipError_t launch_few4(const KArgs& a, int head_dim, int rb, hipStream_t s) {
    if (a.n_items == 0) return hipSuccess;
    if (head_dim == 64) {
        if (rb == 1) return launch_few4_rows<64, 1>(a, s);
        else if (rb == 2) return launch_few4_rows<64, 2>(a, s);
        else return launch_few4_rows<64, 4>(a, s);
    } else {
        if (rb == 1) return launch_few4_rows<128, 1>(a, s);
        else return launch_few4_rows<128, 2>(a, s);
    }
}

hipError_t launch_tables(const TablesArgs& a, hipStream_t s) {
    return launch(tables_kernel, dim3((a.n_items + 15) / 16), dim3(256), a, s);
}

}  // namespace mstar
