// The packed cache in 8 bits: blocks of 32 rows of a segment, one scale for the keys and one for the values of each.
//
// A scale is a power of two (the smallest one that brings the block's largest magnitude to at most 448 for e4m3 and 127 for
// int8, at least 2^-126; 0 for a block of zeros), so that every quotient is exact and a code is one rounding to nearest even
// of the value itself, whatever order the arithmetic has.  Raising a block's scale is a shift with one more rounding, at
// most half a step of the new scale, so that a block whose scale has been raised n times is off by less than one step of
// its last scale.  A code times its scale is exact in fp32.
//
// Block b of segment s has scale number cap[s] / 32 + s + b (cap[s]: the segment's first row).  Segments start at any row, so
// ceil(rows / 32) of them can be one more than their rows' share of a table counted from row 0; the + s makes room for it:
// the numbers of two segments never meet, and no table of block counts is needed.
#pragma once

#include "lkv_common.h"

namespace lkv {

constexpr int kQuantBlock = 32;
constexpr int kQuantE4m3 = 0;
constexpr int kQuantInt8 = 1;

// One side's device pointers of a packed 8-bit cache.
struct QuantRows {
  uint8_t* k;
  uint8_t* v;
  float* k_scale;
  float* v_scale;
};

__device__ __forceinline__ int quant_first_scale(int cap, int s) { return cap / kQuantBlock + s; }

// Scale of a block whose largest finite magnitude is `top`.
template <int kFormat>
__device__ __forceinline__ float quant_scale(float top) {
  const uint32_t bits = __float_as_uint(top);
  const int e = (int)(bits >> 23);
  const uint32_t man = bits & 0x7fffffu;
  // 448 = 1.75 x 2^8 and 127 = 1.984375 x 2^6: one binade more where the mantissa is above theirs
  const int field = kFormat == kQuantE4m3 ? e - 8 + (man > 0x600000u ? 1 : 0) : e - 6 + (man > 0x7e0000u ? 1 : 0);
  return top > 0.f ? __uint_as_float((uint32_t)max(field, 1) << 23) : 0.f;
}

// 1 / scale of a power of two in [2^-126, 2^126], 0 of 0.
__device__ __forceinline__ float quant_inverse(float scale) {
  return scale > 0.f ? __uint_as_float((254u << 23) - __float_as_uint(scale)) : 0.f;
}

// Four values, already divided by their scale, to four codes.
template <int kFormat>
__device__ __forceinline__ uint32_t quant4(float a, float b, float c, float d) {
  if constexpr (kFormat == kQuantE4m3) {
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
    return (uint32_t)r;
  } else {
    // 1.5 x 2^23 more: the low mantissa byte is the whole number in two's complement, rounded to nearest even
    constexpr float kMagic = 12582912.f;
    const uint32_t ua = __float_as_uint(a + kMagic), ub = __float_as_uint(b + kMagic);
    const uint32_t uc = __float_as_uint(c + kMagic), ud = __float_as_uint(d + kMagic);
    const uint32_t lo = __builtin_amdgcn_perm(ub, ua, 0x0c0c0400u), hi = __builtin_amdgcn_perm(ud, uc, 0x0c0c0400u);
    return __builtin_amdgcn_perm(hi, lo, 0x05040100u);
  }
}

// Four codes to the numbers they stand for in units of the scale (exact).
template <int kFormat>
__device__ __forceinline__ void unquant4(uint32_t w, float (&f)[4]) {
  if constexpr (kFormat == kQuantE4m3) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo.x; f[1] = lo.y; f[2] = hi.x; f[3] = hi.y;
  } else {
    f[0] = (float)(int8_t)(w & 0xffu);
    f[1] = (float)(int8_t)(w >> 8 & 0xffu);
    f[2] = (float)(int8_t)(w >> 16 & 0xffu);
    f[3] = (float)(int8_t)(w >> 24);
  }
}

// A value for the codes where the block holds values that are not finite: NaN as 0, infinities as the largest code.
template <int kFormat>
__device__ __forceinline__ float quant_tame(float y) {
  constexpr float kMost = kFormat == kQuantE4m3 ? 448.f : 127.f;
  return y != y ? 0.f : fminf(fmaxf(y, -kMost), kMost);
}

// Largest s in [0, n - 1] with key(s) <= p, for a key that grows with s and key(0) <= p; by the whole wave, 64 probes a round.
template <typename Key>
__device__ __forceinline__ int wave_upper_key(int n, int p, int lane, Key key) {
  int lo = 0, len = n;
  while (len > 1) {
    const int step = (len + 63) >> 6;
    const int i = lo + lane * step;
    const bool le = i < lo + len && key(min(i, n - 1)) <= p;
    const int cnt = max(1, __popcll(__ballot(le)));
    const int new_lo = lo + (cnt - 1) * step;
    len = min(step, lo + len - new_lo);
    lo = new_lo;
  }
  return lo;
}

// Maximum over the 64 lanes of a wave, in every lane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) {
#define LKV_MAX_STEP(ctrl) x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, 0xf, 0xf, true))
  LKV_MAX_STEP(kDppQuadXor1);
  LKV_MAX_STEP(kDppQuadXor2);
  LKV_MAX_STEP(kDppRowHalfMirror);
  LKV_MAX_STEP(kDppRowMirror);
#undef LKV_MAX_STEP
  const u32x2_swap_t a = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = max(a.x, a.y);
  const u32x2_swap_t b = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return max(b.x, b.y);
}

}  // namespace lkv
