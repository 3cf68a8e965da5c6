// Device code shared by the kernels over caches held in 4 or 8 bits: elements to bf16 and
// back.
//
// gfx950 converts two elements of either format to bf16, times a power of two, in one
// instruction of the plain vector rate (5.0 clocks per wavefront and instruction, as a
// multiply-add), so that a row in 4 bits costs half an instruction per element where
// integers with a scale take a shift, a mask and a multiply each.  The instruction takes
// bits 30:23 of its scale operand and nothing else of it, and gives NaN for 255.
#pragma once

#include "device_common.h"
#include "internal.h"

namespace spec {

// A row of a head: 4 lanes' parts of 32 elements, one group each.
constexpr int kGroup = 32;
template <int BITS>
struct RowPart {                // 32 elements
  uint4 w[BITS / 4];
};
constexpr int part_bytes(int bits) { return kGroup * bits / 8; }

// Byte i of `bytes`, as a scale operand: 2^(byte - 127), NaN for 255.
__device__ __forceinline__ float scale_of(uint32_t bytes, int i) {
  return __uint_as_float((bytes >> (8 * i)) << 23);
}

// Elements 8 s .. 8 s + 7 of a part.
template <int BITS>
__device__ __forceinline__ bf16x8 elements8(const RowPart<BITS>& r, int s, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 e[4];
  if constexpr (BITS == 4) {
    const uint32_t w = s == 0 ? r.w[0].x : s == 1 ? r.w[0].y : s == 2 ? r.w[0].z : r.w[0].w;
    e[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    e[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
    e[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
    e[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  } else {
    const uint4 q = r.w[s / 2 * (BITS / 8)];
    const uint32_t w0 = s % 2 == 0 ? q.x : q.z, w1 = s % 2 == 0 ? q.y : q.w;
    e[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false);
    e[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true);
    e[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false);
    e[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true);
  }
  return bf16x8{e[0][0], e[0][1], e[1][0], e[1][1], e[2][0], e[2][1], e[3][0], e[3][1]};
}

// Elements i .. i + 3 of a row (i a multiple of 4), in 32 bits.
template <int BITS>
__device__ __forceinline__ floatx4 elements4(const uint8_t* row, int i, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 a, b;
  if constexpr (BITS == 4) {
    const uint32_t w = *reinterpret_cast<const uint16_t*>(row + i / 2);
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  } else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(row + i);
    a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
    b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
  }
  return floatx4{(float)a[0], (float)a[1], (float)b[0], (float)b[1]};
}

// The scale byte of a group whose largest magnitude has the bf16 bits `top`: X + 127
// with X the least that has top <= 1.75 2^(X + E), E = 2 (4 bits) or 8: a mantissa
// above .75 carries into the exponent.
template <int BITS>
__device__ __forceinline__ int scale_byte(uint32_t top) {
  if (top >= 0x7f80u) return 255;
  const int x = (int)((top + 0x1fu) >> 7) - (BITS == 4 ? 2 : 8);
  return clampi(x, 127 - 111, 127 + (BITS == 4 ? 125 : 119));
}

// Two bf16 to elements of their group, placed at byte (4 bits) or half (8 bits) `AT` of w.
// The instructions round to nearest, ties to even; that to 4 bits saturates, that to 8
// does not, so that magnitudes are held at the largest element's for the largest scale
// (the only one that does not follow from the group's magnitude): 448 2^119.
template <int BITS, int AT>
__device__ __forceinline__ uint32_t elements2(uint32_t w, uint32_t x, float scale) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  typedef short shortx2 __attribute__((ext_vector_type(2)));
  if constexpr (BITS == 4) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(bf16x2, x), scale, AT);
  } else {
    typedef uint16_t ushortx2 __attribute__((ext_vector_type(2)));
    const ushortx2 mag = __builtin_bit_cast(ushortx2, x & 0x7fff7fffu);
    const ushortx2 most = {0x7f60, 0x7f60};
    const uint32_t y = __builtin_bit_cast(uint32_t, __builtin_elementwise_min(mag, most)) |
                       (x & 0x80008000u);
    const shortx2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(
        __builtin_bit_cast(shortx2, w), __builtin_bit_cast(bf16x2, y), scale, AT != 0);
    return __builtin_bit_cast(uint32_t, r);
  }
}

}  // namespace spec
