// Block-scaled ("microscaled") values: blocks of 32 consecutive columns share a
// power-of-two scale 2^(s - 127) held in one byte (s = 255: the block is NaN);
// the values themselves are E2M1 (4 bits, largest 6) or E4M3 (8 bits, largest
// 448).  The formats are those of the OCP Microscaling Formats specification.
//
// A matrix [rows, cols] is held as two arrays:
//   codes  [rows, pitch]: cols rounded up to whole groups of 256 columns; E4M3
//          one byte a column, E2M1 two columns a byte (the even column in the
//          low half).  Columns past cols are zeros, so a product may run over
//          whole groups.
//   scales [groups, slots, 8], slots = rows rounded up to 32: the eight scales of
//          a row's group together, then the next row's, so that a product's
//          tile finds the scales of a group of columns in one run of memory
//          (beside the row-major codes they would be 8 bytes of every line).
#pragma once

#include "common.h"

namespace dlmc {

constexpr int MX_BLOCK = 32, MX_GROUP = 256;

inline int mx_groups(int cols) { return ceil_div(cols, MX_GROUP); }
inline size_t mx_slots(int64_t rows) { return ((size_t)rows + 31) & ~(size_t)31; }
// bytes of a row of codes
inline size_t mx_pitch(int fmt, int cols) { return (size_t)mx_groups(cols) * (fmt == DLMC_MX_FP4 ? 128 : 256); }
inline size_t mx_code_bytes(int fmt, int64_t rows, int cols) { return (size_t)rows * mx_pitch(fmt, cols); }
inline size_t mx_scale_bytes(int64_t rows, int cols) { return mx_slots(rows) * 8 * (size_t)mx_groups(cols); }

struct MxView {
  uint8_t* codes = nullptr;
  uint8_t* scales = nullptr;
};

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)

// The scale's byte of a block whose largest magnitude has the bits `top` (sign
// cleared): the least power of two 2^e, e >= -127, with top <= F 2^e, F = 6
// = 1.5 2^2 or 448 = 1.75 2^8, so no value of the block saturates and each is off
// by at most half a step of its own binade.  Adding 2^23 - 1 - (fraction of F)
// carries into the exponent exactly where the fraction of top exceeds F's.  An
// infinity or NaN in the block gives 255.
template <int FMT>
__device__ __forceinline__ uint32_t mx_scale_code(uint32_t top) {
  constexpr uint32_t CARRY = FMT == DLMC_MX_FP4 ? 0x3FFFFFu : 0x1FFFFFu;
  constexpr int EMAX = FMT == DLMC_MX_FP4 ? 2 : 8;
  const int e = (int)((top + CARRY) >> 23) - EMAX;
  return top >= 0x7F800000u ? 255u : (uint32_t)max(e, 0);
}

// lane's value of lane ^ 1 and lane ^ 2 (within four lanes) by DPP moves
template <int CTRL>
__device__ __forceinline__ uint32_t mx_dpp(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
#else
  return x;
#endif
}

// Eight columns of a block by each of four neighbouring lanes (all four of them
// active): this lane's codes, E4M3 in lo, hi, E2M1 in lo; returns the scale's
// byte.  The scaling is a product with a power of two, exact but below 2^-126,
// where the code is zero either way; the conversions round to nearest even.
template <int FMT>
__device__ __forceinline__ uint32_t mx_encode8(const float (&v)[8], uint32_t& lo, uint32_t& hi) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, v[i]) & 0x7FFFFFFFu);
  top = max(top, mx_dpp<0xB1>(top));
  top = max(top, mx_dpp<0x4E>(top));
  const uint32_t s = mx_scale_code<FMT>(top);
  lo = hi = 0;
#if defined(__HIP_DEVICE_COMPILE__)
  if (s != 255u) {
    const float inv = __builtin_bit_cast(float, (254u - s) << 23);
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = v[i] * inv;
    if constexpr (FMT == DLMC_MX_FP4) {
      lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(lo, w[0], w[1], 1.0f, 0);
      lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(lo, w[2], w[3], 1.0f, 1);
      lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(lo, w[4], w[5], 1.0f, 2);
      lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(lo, w[6], w[7], 1.0f, 3);
    } else {
      lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[0], w[1], (int)lo, false);
      lo = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[2], w[3], (int)lo, true);
      hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[4], w[5], (int)hi, false);
      hi = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(w[6], w[7], (int)hi, true);
    }
  }
#endif
  return s;
}

// Eight codes' values: E4M3 from lo, hi, E2M1 from lo; s is their scale's byte.
template <int FMT>
__device__ __forceinline__ void mx_decode8(uint32_t lo, uint32_t hi, uint32_t s, float (&v)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  f32x2 p[4];
  if constexpr (FMT == DLMC_MX_FP4) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(lo, 1.0f, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(lo, 1.0f, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(lo, 1.0f, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(lo, 1.0f, 3);
  } else {
    p[0] = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, false);
    p[1] = __builtin_amdgcn_cvt_pk_f32_fp8((int)lo, true);
    p[2] = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, false);
    p[3] = __builtin_amdgcn_cvt_pk_f32_fp8((int)hi, true);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = ldexpf(p[i / 2][i % 2], (int)s - 127);
    v[i] = s == 255u ? __builtin_nanf("") : x;
  }
#endif
}

#endif  // device helpers

}  // namespace dlmc
