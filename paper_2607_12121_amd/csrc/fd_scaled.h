// 8-bit values with block scales: e4m3 codes (largest 448) times 2^(s - 127), s one byte (E8M0)
// per block of 128 columns of a row (activations) or of 128 x 128 (weights).
//
// The scale is the least power of two at which the block's largest magnitude is at most 448.  A
// power of two costs a floating code nothing (the relative rounding of e4m3, 2^-4, does not depend
// on it; only values more than 2^15 below the block's largest lose bits), dividing by it is exact,
// and v_mfma_scale_f32_16x16x128_f8f6f4 applies it inside the matrix instruction.
#pragma once

#include "fd_common.h"

namespace fd {

constexpr int kScaleBlock = 128;

// Bytes between the scale rows of `cols` columns: a byte per block, padded to whole 4-byte words
// (the product reads the scales of four blocks with one load).
__host__ __device__ inline int scale_stride(int cols) { return (cols / kScaleBlock + (cols % kScaleBlock != 0) + 3) & ~3; }

// |x| as ordered bits: the integer maximum of these is the largest magnitude, and infinities and
// NaN come out on top (which a float maximum would drop).
FD_DEVICE uint32_t mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// Scale byte of a block whose largest magnitude has the bits `top`; 255 (NaN) where the block
// holds an infinity or a NaN.  448 = 1.75 * 2^8: the exponent of `top` less 8, one more above
// 1.75.  At least 1, so that the scale is a normal float (a block of zeros has 1).
FD_DEVICE uint32_t scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = static_cast<int>(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
  return static_cast<uint32_t>(e < 1 ? 1 : e);
}
// 1 / 2^(s - 127), exact (a byte from finite values is at most 247); NaN for the NaN byte, so that
// every code of such a block is NaN.
FD_DEVICE float scale_inverse(uint32_t s) { return s == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float((254u - s) << 23); }

// Four floats to four e4m3 codes, round to nearest even; magnitudes are at most 448.
FD_DEVICE uint32_t pack_codes(float a, float b, float c, float d) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return static_cast<uint32_t>(r);
}

// Eight values of a lane to codes: the 16 lanes that share a block (lane & ~15) agree on its
// scale byte, which is returned.  Lanes past the row's end pass zeros.
FD_DEVICE uint32_t quant_lane8(const float (&v)[8], uint2& codes) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, mag_bits(v[e]));
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, kWave)));
  const uint32_t s = scale_byte(top);
  const float inv = scale_inverse(s);
  codes.x = pack_codes(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
  codes.y = pack_codes(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv);
  return s;
}

// GELU, tanh form: z / (1 + 2^-t), t = 2 sqrt(2 / pi) log2(e) (z + 0.044715 z^3), in seven instructions with the
// hardware's exponent and reciprocal (an ulp each); gelu_tanh_fast, whose bits the bf16 products keep, takes two more.
FD_DEVICE float gelu(float z) {
  const float t = z * fmaf(z * z, -0.10294324f, -2.3022082f);
  return z * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(t));
}

FD_DEVICE void unpack_bf8(const uint4 x, float (&v)[8]) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

}  // namespace fd
