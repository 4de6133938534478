// Rows of a quantised cache: blocks of 32 neighbouring dims of one token and KV head, each
// with a power of two of its own, and what the kernels that write and read them share.
//
//   value = code * 2^(s - 127),  s: the block's scale byte; s = 255: the block is NaN
//   e4m3: 8 bits a value, largest 448;  e2m1: 4 bits, largest 6, dim 2 i the low half of byte i
//
// s is the least power of two for which no value is further from its code than half a step of the
// block's largest ones: with A the largest size, A <= 464 * 2^(s - 127) (e4m3: 448 is the
// nearest up to there) or 7 * 2^(s - 127) (e2m1: 6 is), found in the bits of A: raised by what lifts a
// fraction past 1.8125 or 1.75 into the exponent, of which the largest code's exponent is
// taken.  Multiplying by 2^(127 - s) is exact, so that each value is rounded once, to the nearest
// code and the even one in the middle, as the conversion instruction does; what stands for it
// is exact in bf16 as well.  s is at least 10 (2^-117), so that no value stands below fp32's normal
// range, and a block with a size of 2^127 or more, an infinity or NaN has s = 255.  (Of pages from elsewhere, e4m3 under s = 0, 1
// and 2 has values below bf16's smallest, 2^-133: they become the nearest multiple of it, except in fp32.)
#pragma once

#include "serve.h"

namespace gkv {

constexpr int Q_BLOCK = 32;
constexpr uint32_t Q_NONE = 255;

template <int FMT> constexpr int code_bits() { return FMT == GRACEKV_E4M3 ? 8 : 4; }

// byte of (token `at` of page `id`, KV head g, dim 0), and of its scales
template <int FMT> __device__ __forceinline__ int64_t code_row(const PageDims& pg, const QuantDims& qd, int64_t id, int g, int at) {
  return id * qd.code_stride + (((int64_t)g << pg.shift) + at) * (pg.d * code_bits<FMT>() / 8);
}
__device__ __forceinline__ int64_t scale_row(const PageDims& pg, const QuantDims& qd, int64_t id, int g, int at) {
  return id * qd.scale_stride + (((int64_t)g << pg.shift) + at) * (pg.d / Q_BLOCK);
}

// the scale byte of a block whose largest size is `top` (NaN where one of its values is)
template <int FMT> __device__ __forceinline__ uint32_t block_scale(float top) {
  constexpr uint32_t LIFT = FMT == GRACEKV_E4M3 ? 0x17ffffu : 0x1fffffu;
  constexpr int EMAX = FMT == GRACEKV_E4M3 ? 8 : 2;
  const uint32_t bits = __float_as_uint(top);
  if (bits >= 0x7f000000u) return Q_NONE;                    // 2^127 and up
  const int s = (int)((bits + LIFT) >> 23) - EMAX;
  return (uint32_t)max(s, 10);
}
// 2^(127 - s)
__device__ __forceinline__ float unscale(uint32_t s) { return __uint_as_float((254u - min(s, 254u)) << 23); }
// 2^(s - 127) as the conversions take it: they go by its exponent, 255 being NaN
__device__ __forceinline__ float scale_of(uint32_t s) { return __uint_as_float(s << 23); }

typedef __bf16 q_bf16x2 __attribute__((ext_vector_type(2)));

// Codes of eight values, times 2^(127 - s) already: two words (e4m3) or one.
template <int FMT> struct Codes8 { uint32_t w[FMT == GRACEKV_E4M3 ? 2 : 1]; };
template <int FMT> __device__ __forceinline__ Codes8<FMT> to_codes(const float* x) {
  Codes8<FMT> c;
  if constexpr (FMT == GRACEKV_E4M3) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f);       // past it the conversion gives NaN
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h], y[4 * h + 1], 0, false);
      c.w[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2], y[4 * h + 3], lo, true);
    }
  } else {                                                   // saturates by itself
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], 1.f, 3);
    c.w[0] = w;
  }
  return c;
}

// Two neighbouring values, number P of the pairs in a word (0, 1; e2m1: 0 .. 3), as bf16
template <int FMT, int P> __device__ __forceinline__ uint32_t pair_bf16(uint32_t w, float scale) {
  if constexpr (FMT == GRACEKV_E4M3)
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, P == 1));
  else
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, P));
}
// eight values, from the words that hold them
template <int FMT> __device__ __forceinline__ uint4 eight_bf16(const uint32_t* w, float scale) {
  if constexpr (FMT == GRACEKV_E4M3)
    return make_uint4(pair_bf16<FMT, 0>(w[0], scale), pair_bf16<FMT, 1>(w[0], scale), pair_bf16<FMT, 0>(w[1], scale),
                      pair_bf16<FMT, 1>(w[1], scale));
  else
    return make_uint4(pair_bf16<FMT, 0>(w[0], scale), pair_bf16<FMT, 1>(w[0], scale), pair_bf16<FMT, 2>(w[0], scale),
                      pair_bf16<FMT, 3>(w[0], scale));
}

// eight values as floats, from the words that hold them
template <int FMT> __device__ __forceinline__ void eight_f32(const uint32_t* w, float scale, float* x) {
  f32x2 p[4];
  if constexpr (FMT == GRACEKV_E4M3) {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], scale, false);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[0], scale, true);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[1], scale, false);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w[1], scale, true);
  } else {
    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 0);
    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 1);
    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 2);
    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w[0], scale, 3);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = p[i / 2][i & 1];
}

// the kernel's template arguments from the shapes
template <typename F> inline void by_type(const PageDims& pg, int format, F go) {
  using std::integral_constant;
  auto dims = [&](auto type) {
    auto codes = [&](auto dim) {
      if (format == GRACEKV_E4M3) go(type, dim, integral_constant<int, GRACEKV_E4M3>{});
      else go(type, dim, integral_constant<int, GRACEKV_E2M1>{});
    };
    if (pg.d == 128) codes(integral_constant<int, 128>{}); else codes(integral_constant<int, 64>{});
  };
  if (pg.dtype == GRACEKV_BF16) dims(uint16_t{}); else dims(float{});
}

}  // namespace gkv
