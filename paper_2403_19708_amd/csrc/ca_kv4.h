// The 4-bit cache: layout and the device helpers that read and write it.
//
// A row is the D values of one token and kv head.  Every 32 of them have a scale byte e, which stands for 2^(e - 127), and a value is
// that times its e2m1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign).  Scale bytes from 253 on stand for NaN (6 * 2^126 is no bf16 number).
// Two codes a byte, the first in the low half.  gfx950 converts pairs of codes with their scale in one instruction, exactly for every
// scale from 0 to 252.
//   page of a head (Kv4<D>::kBlock bytes): 16 rows of codes, then 16 rows of scale bytes
//   row of the tier (kv4_row_bytes): the codes of all kv heads, then their scale bytes, zeros up to a multiple of 16
#pragma once

#include "ca_device.h"

namespace ca {

namespace {

constexpr uint32_t kKv4MostScale = 252;

template <int D>
struct Kv4 {
    static constexpr int kCodes = D / 2;                                  // bytes of a row
    static constexpr int kScales = D / 32;
    static constexpr int kScaleAt = kPageSize * kCodes;                   // inside a page of a head
    static constexpr int kBlock = kPageSize * (kCodes + kScales);
};

__device__ inline bool kv4_is_nan(uint32_t e) { return e > kKv4MostScale; }
__device__ inline float kv4_scale(uint32_t e) { return __uint_as_float(e << 23); }      // as the conversions take it (0: 2^-127)
// the largest of a key's scale bytes that are numbers
template <int D>
__device__ __attribute__((always_inline)) inline uint32_t kv4_most_scale(uint32_t e) {
    uint32_t most = 0;
#pragma unroll
    for (int b = 0; b < D / 32; ++b) {
        const uint32_t one = e >> 8 * b & 255u;
        most = max(most, kv4_is_nan(one) ? 0u : one);
    }
    return most;
}

// codes of a word -> values 2 i and 2 i + 1
__device__ __attribute__((always_inline)) inline float2 pair_f32(uint32_t w, float scale, int i) {
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    f32x2 v;
    switch (i) {
        case 0: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0); break;
        case 1: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1); break;
        case 2: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2); break;
        default: v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3); break;
    }
    return make_float2(v[0], v[1]);
}
__device__ __attribute__((always_inline)) inline uint32_t pair_bf16(uint32_t w, float scale, int i) {
    bf16x2 v;
    switch (i) {
        case 0: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0); break;
        case 1: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1); break;
        case 2: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2); break;
        default: v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3); break;
    }
    return __builtin_bit_cast(uint32_t, v);
}

typedef __attribute__((ext_vector_type(2))) _Float16 half2v;
typedef __attribute__((ext_vector_type(8))) _Float16 half8v;

__device__ inline uint32_t pack_f16(float lo, float hi) { return __builtin_bit_cast(uint32_t, half2v{(_Float16)lo, (_Float16)hi}); }

__device__ __attribute__((always_inline)) inline half2v pair_f16(uint32_t w, float scale, int i) {
    switch (i) {
        case 0: return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 0));
        case 1: return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 1));
        case 2: return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 2));
        default: return __builtin_bit_cast(half2v, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, scale, 3));
    }
}

// Two dims of either half of a row, rotated in packed fp16: word w of a lane's c and s (W words each, for 2 W dims of either half).  Style 0: the pairs
// are lo[i], hi[i]; 1: the two of lo, the two of hi (pairs of the lower half, then of the upper half in c and s).
template <int STYLE, int W>
__device__ __attribute__((always_inline)) inline void rotate_pair(half2v &lo, half2v &hi, const uint32_t (&c)[W], const uint32_t (&s)[W], int w) {
    if (STYLE == 0) {
        const half2v cc = __builtin_bit_cast(half2v, c[w]), ss = __builtin_bit_cast(half2v, s[w]);
        const half2v l = lo * cc - hi * ss;
        hi = hi * cc + lo * ss;
        lo = l;
    } else {
        const half2v c0 = __builtin_bit_cast(half2v, c[w / 2]), s0 = __builtin_bit_cast(half2v, s[w / 2]);
        const half2v c1 = __builtin_bit_cast(half2v, c[W / 2 + w / 2]), s1 = __builtin_bit_cast(half2v, s[W / 2 + w / 2]);
        const half2v ca_ = w % 2 ? half2v{c0[1], c0[1]} : half2v{c0[0], c0[0]}, cb_ = w % 2 ? half2v{c1[1], c1[1]} : half2v{c1[0], c1[0]};
        const half2v sa = w % 2 ? half2v{-s0[1], s0[1]} : half2v{-s0[0], s0[0]}, sb = w % 2 ? half2v{-s1[1], s1[1]} : half2v{-s1[0], s1[0]};
        lo = lo * ca_ + half2v{lo[1], lo[0]} * sa;
        hi = hi * cb_ + half2v{hi[1], hi[0]} * sb;
    }
}

// Eight values of either half of a query row (16-byte pieces `piece` and `piece` + D/16), normalised, rotated, times f, as fp16.  The D / 16
// lanes that share a row are neighbours and all active.  Returns the factor to multiply by: 1 but for rows whose largest value would leave
// the middle of fp16's range, which are scaled to at most 1 by a power of two.
template <int D, int STYLE>
__device__ __attribute__((always_inline)) inline float query_pieces(const AttnArgs &a, const uint16_t *row, int pos, int piece, float f, uint4 &x, uint4 &y) {
    constexpr int HALF = D / 2;
    x = *reinterpret_cast<const uint4 *>(row + 8 * piece);
    y = *reinterpret_cast<const uint4 *>(row + HALF + 8 * piece);
    float2 cs[8];
    load_cs<D, STYLE>(a.rope, pos, piece, cs);
    uint32_t *px = reinterpret_cast<uint32_t *>(&x), *py = reinterpret_cast<uint32_t *>(&y);
    float of[16];                                        // eight of either half
    float *const u = of, *const v = of + 8;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        u[2 * w] = bf_lo(px[w]); u[2 * w + 1] = bf_hi(px[w]);
        v[2 * w] = bf_lo(py[w]); v[2 * w + 1] = bf_hi(py[w]);
    }
    if (a.q_weight) {
        const float inv = head_norm<D, D / 16>(of, a.norm_eps);
        const uint4 gx = *reinterpret_cast<const uint4 *>(a.q_weight + 8 * piece), gy = *reinterpret_cast<const uint4 *>(a.q_weight + HALF + 8 * piece);
        const uint32_t *wx = reinterpret_cast<const uint32_t *>(&gx), *wy = reinterpret_cast<const uint32_t *>(&gy);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            u[2 * w] *= inv * bf_lo(wx[w]); u[2 * w + 1] *= inv * bf_hi(wx[w]);
            v[2 * w] *= inv * bf_lo(wy[w]); v[2 * w + 1] *= inv * bf_hi(wy[w]);
        }
    }
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        u[i] *= f;
        v[i] *= f;
        most = fmaxf(most, fmaxf(fabsf(u[i]), fabsf(v[i])));
    }
#pragma unroll
    for (int m = 1; m < D / 16; m *= 2) most = fmaxf(most, __shfl_xor(most, m));
    const int exponent = (int)(__float_as_uint(most) >> 23) - 126;       // most <= 2^exponent
    const int up = most == 0.f || (exponent > -6 && exponent < 12) ? 0 : min(max(exponent, -100), 127);
    if (up != 0)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            u[i] = __builtin_ldexpf(u[i], -up);
            v[i] = __builtin_ldexpf(v[i], -up);
        }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (STYLE == 0) {
            const float2 c0 = cs[2 * w], c1 = cs[2 * w + 1];
            px[w] = pack_f16(u[2 * w] * c0.x - v[2 * w] * c0.y, u[2 * w + 1] * c1.x - v[2 * w + 1] * c1.y);
            py[w] = pack_f16(v[2 * w] * c0.x + u[2 * w] * c0.y, v[2 * w + 1] * c1.x + u[2 * w + 1] * c1.y);
        } else {
            const float2 c0 = cs[w], c1 = cs[4 + w];
            px[w] = pack_f16(u[2 * w] * c0.x - u[2 * w + 1] * c0.y, u[2 * w + 1] * c0.x + u[2 * w] * c0.y);
            py[w] = pack_f16(v[2 * w] * c1.x - v[2 * w + 1] * c1.y, v[2 * w + 1] * c1.x + v[2 * w] * c1.y);
        }
    }
    return __builtin_ldexpf(1.0f, up);
}

}  // namespace

}  // namespace ca
