// Device code of the 4-bit cache: where a record keeps a key's codes and
// scales, and how codes become bf16 values.  The layout is that of
// mstar_cache.h; in a wave's terms (lane l = 16 G + n) a lane's D / 8 bytes of
// a record are, for K, dims [G D / 4, (G + 1) D / 4) of key n, and for V, dims
// [n D / 16, (n + 1) D / 16) of keys 4 G .. 4 G + 3.
#pragma once
#include "cache.h"
#include "device.h"

namespace mstar {
namespace {

typedef bf16_t bf16x2 __attribute__((ext_vector_type(2)));

constexpr int MSTAR_DEVERR_NONFINITE_BIT = MSTAR_DEVERR_NONFINITE;
constexpr int kScaleMin = 2, kScaleMax = 252;  // scale bytes: every value is a normal, finite bf16 number

template <int D>
struct Record {
    static constexpr int kBytes = MSTAR_KV4_RECORD_BYTES(D);
    static constexpr int kScales = 8 * D;   // offset of the scale bytes
    static constexpr int kWord = D / 32;    // bytes of D / 16 dims of one key: what lane n holds of a row
    // word n (dims [n D / 16, +D / 16)) of key `slot`
    __device__ __forceinline__ static int k_word(int slot, int n) {
        return ((n >> 2) * 16 + slot) * (D / 8) + (n & 3) * kWord;
    }
    __device__ __forceinline__ static int v_word(int slot, int n) {
        return (((slot >> 2) * 16 + n) * 4 + (slot & 3)) * kWord;
    }
    __device__ __forceinline__ static int scale(int slot, int n) { return kScales + (n * (D / 16) / 32) * 16 + slot; }
};

// The scale byte as the fp32 operand of the conversions, which use its exponent.
__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Byte B of `w` as two bf16 values.
template <int B>
__device__ __forceinline__ bf16x2 pair_of(uint32_t w, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, B);
}

// Four bytes of `w` as eight bf16 values; two from byte B on as four.
__device__ __forceinline__ bf16x8 eight_of(uint32_t w, float scale) {
    const bf16x2 a = pair_of<0>(w, scale), b = pair_of<1>(w, scale), c = pair_of<2>(w, scale), d = pair_of<3>(w, scale);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <int B>
__device__ __forceinline__ bf16x4 four_of(uint32_t w, float scale) {
    const bf16x2 a = pair_of<B>(w, scale), b = pair_of<B + 1>(w, scale);
    return bf16x4{a[0], a[1], b[0], b[1]};
}

// softmax_update with the maximum across a row's four lanes taken only when the
// reference has to move: a lane compares its own scores with the reference, and
// none exceeding it by kLazy means that no row's maximum does.  The same results,
// without the cross-lane exchange in almost every step.
template <int RB, int NB>
__device__ __forceinline__ bool softmax_lazy(const RowGroup& rg, f32x4 (&s)[RB][NB], float c, float (&m)[RB],
                                             float (&l)[RB], float (&alpha)[RB]) {
    float mx[RB];
    bool grow = false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        mx[rb] = tree_max<NB>(s[rb]) * c;
        grow |= mx[rb] > m[rb] + kLazy;
    }
    const bool rescale = __builtin_amdgcn_ballot_w64(grow) != 0;
    float m_use[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        alpha[rb] = 1.0f;
        if (rescale) {
            const float m_new = fmax_num(m[rb], rg.max(mx[rb]));
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
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const float sum = tree_sum<NB>(s[rb]);
        l[rb] = rescale ? l[rb] * alpha[rb] + sum : l[rb] + sum;
    }
    return rescale;
}

// Dims 2 b and 2 b + 1 of the D / 16 that a lane's V codes `v` hold of key j.
template <int D>
__device__ __forceinline__ bf16x2 v_pair(const uint32_t* v, int j, int b, float scale) {
    const int byte = D == 128 ? b : 2 * (j & 1) + b;
    const uint32_t w = v[D == 128 ? j : j >> 1];
    return byte == 0 ? pair_of<0>(w, scale) : byte == 1 ? pair_of<1>(w, scale) : byte == 2 ? pair_of<2>(w, scale)
                                                                              : pair_of<3>(w, scale);
}

// Scale byte j of the four in `w`, at most the largest that a stored row has: a
// hidden key's probability is 0, and 0 times what any byte up to that one stands
// for is 0, where an infinity would reach rows that do not see the key.
__device__ __forceinline__ uint32_t v_scale(uint32_t w, int j) { return min((w >> (8 * j)) & 0xffu, (uint32_t)kScaleMax); }

}  // namespace
}  // namespace mstar
