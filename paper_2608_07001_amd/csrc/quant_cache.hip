// New tokens into a quantised paged cache, keys rotated to their position on the way, and rows
// of it back.
//
//   K[place] <- Q(R(pos) k),  V[place] <- Q(v),  q_out <- R(pos) q      (quant.h for Q)
//   R(p): (x_i, x_{i + d/2}) -> (x_i c - x_{i+d/2} s, x_{i+d/2} c + x_i s), row p of the tables
//   k[row] <- what K[place] stands for,  v[row] likewise
//
// A rotated key is quantised from fp32, where its two products and their sum are each rounded
// (no fused multiply and add: the same codes wherever the rotation is formed like that), and
// not rounded to the rows' type before.  Reading back is exact in bf16 and fp32.
#include "quant.h"

namespace gkv {

constexpr int QC_T = 256;

// eight neighbouring elements of a row as floats
template <typename T> struct Eight;
template <> struct Eight<uint16_t> {
  uint4 u;
  __device__ __forceinline__ void load(const uint16_t* p) { u = *(const uint4*)p; }
  __device__ __forceinline__ void get(float* x) const {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ void put(uint16_t* p, const float* x) {
    *(uint4*)p = make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
};
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const float4*)p; b = *(const float4*)(p + 4); }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void put(float* p, const float* x) {
    *(float4*)p = make_float4(x[0], x[1], x[2], x[3]);
    *(float4*)(p + 4) = make_float4(x[4], x[5], x[6], x[7]);
  }
};

// Largest size of 32 values, eight on each of four neighbouring lanes.  Sizes are compared by
// their bits, under which NaN is the largest.
__device__ __forceinline__ float block_top(const float* x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(x[i]) & 0x7fffffffu);
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xf, 0xf, true));      // quad_perm 1, 0, 3, 2
  m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xf, 0xf, true));      // quad_perm 2, 3, 0, 1
  return __uint_as_float(m);
}

// eight values of a block to their codes at `to` and, by the block's first lane, the scale
template <int FMT> __device__ __forceinline__ void put_codes(const float* x, uint8_t* to, uint8_t* scale, bool first) {
  const uint32_t s = block_scale<FMT>(block_top(x));
  const float f = unscale(s);
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = s == Q_NONE ? 0.f : x[i] * f;
  const Codes8<FMT> c = to_codes<FMT>(y);
  if constexpr (FMT == GRACEKV_E4M3) *(uint2*)to = make_uint2(c.w[0], c.w[1]);
  else *(uint32_t*)to = c.w[0];
  if (first) *scale = (uint8_t)s;
}

template <typename T, int D, int FMT>
__global__ __launch_bounds__(QC_T) void k_quant_append(PageDims pg, QuantDims qd, AppendDims ap, const T* __restrict__ k,
                                                       const T* __restrict__ v, const T* q, const int32_t* __restrict__ table,
                                                       const int32_t* __restrict__ start, const int32_t* __restrict__ cu,
                                                       const int32_t* __restrict__ pos, const float* __restrict__ cosT,
                                                       const float* __restrict__ sinT, T* q_out) {
#pragma clang fp contract(off)
  constexpr int U = D / 16;                            // lanes of a head: eight dims of either half
  const int64_t t = blockIdx.x;
  const int unit = blockIdx.y * QC_T + threadIdx.x;
  const int slot = unit / U, c = (unit % U) * 8;       // slot: K heads, V heads, query heads
  const int b = find_span(cu, pg.n_seq, t);
  const Span sp = span_of(cu, b, ap.n_new);
  if (t < sp.a || t >= sp.a + sp.n) return;            // behind the last sequence
  const int64_t place = (int64_t)start[b] + (t - sp.a);
  if (place < 0 || place >= ((int64_t)pg.width << pg.shift)) return;
  const int64_t p = pos ? pos[t] : 0;
  if (pos && (p < 0 || p >= ap.rope_rows)) return;
  const int64_t id = table[(int64_t)b * pg.width + (place >> pg.shift)];
  const int at = (int)(place & (((int64_t)1 << pg.shift) - 1));
  if (id < 0 || id >= pg.n_pages) return;
  if (slot >= 2 * pg.G + (q ? pg.H : 0)) return;
  const bool key = slot < pg.G, value = !key && slot < 2 * pg.G;
  const int head = key ? slot : (value ? slot - pg.G : slot - 2 * pg.G);
  const T* src = key ? k + t * ap.k_tok + head * ap.k_head : (value ? v + t * ap.v_tok + head * ap.v_head : q + t * ap.q_tok + head * ap.q_head);
  Eight<T> lo, hi;
  lo.load(src + c);
  hi.load(src + c + D / 2);
  float x[8], y[8];
  lo.get(x);
  hi.get(y);
  if (pos && !value) {
#pragma unroll
    for (int i = 0; i < 8; i += 4) {
      const float4 fc = *(const float4*)(cosT + p * (D / 2) + c + i), fs = *(const float4*)(sinT + p * (D / 2) + c + i);
      const float cs[4] = {fc.x, fc.y, fc.z, fc.w}, sn[4] = {fs.x, fs.y, fs.z, fs.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a = x[i + j], e = y[i + j];
        x[i + j] = a * cs[j] - e * sn[j];
        y[i + j] = e * cs[j] + a * sn[j];
      }
    }
  }
  if (key || value) {
    uint8_t* codes = (key ? qd.K : qd.V) + code_row<FMT>(pg, qd, id, head, at);
    uint8_t* scales = (key ? qd.Ks : qd.Vs) + scale_row(pg, qd, id, head, at);
    constexpr int B = code_bits<FMT>();
    const bool first = c % Q_BLOCK == 0;
    put_codes<FMT>(x, codes + c * B / 8, scales + c / Q_BLOCK, first);
    put_codes<FMT>(y, codes + (c + D / 2) * B / 8, scales + (c + D / 2) / Q_BLOCK, first);
  } else {
    T* dst = q_out + t * ap.o_tok + head * ap.o_head;
    Eight<T>::put(dst + c, x);
    Eight<T>::put(dst + c + D / 2, y);
  }
}

template <typename T, int D, int FMT>
__global__ __launch_bounds__(QC_T) void k_quant_read(PageDims pg, QuantDims qd, ReadDims rd, const int32_t* __restrict__ table,
                                                     const int32_t* __restrict__ start, const int32_t* __restrict__ cu,
                                                     T* __restrict__ k, T* __restrict__ v) {
  constexpr int U = D / 8;                             // lanes of a head: eight dims
  const int64_t t = blockIdx.x;
  const int unit = blockIdx.y * QC_T + threadIdx.x;
  const int slot = unit / U, c = (unit % U) * 8;
  const int b = find_span(cu, pg.n_seq, t);
  const Span sp = span_of(cu, b, rd.n_rows);
  if (t < sp.a || t >= sp.a + sp.n) return;
  if (slot >= 2 * pg.G) return;
  const int64_t place = (int64_t)start[b] + (t - sp.a);
  int64_t id = -1;
  if (place >= 0 && place < ((int64_t)pg.width << pg.shift)) id = table[(int64_t)b * pg.width + (place >> pg.shift)];
  const int at = (int)(place & (((int64_t)1 << pg.shift) - 1));
  const bool key = slot < pg.G;
  if (key ? !k : !v) return;
  const int head = key ? slot : slot - pg.G;
  T* dst = key ? k + t * rd.k_tok + head * rd.k_head : v + t * rd.v_tok + head * rd.v_head;
  uint4 x = make_uint4(0, 0, 0, 0);                    // no page: nothing is there
  if (id >= 0 && id < pg.n_pages) {
    const uint8_t* codes = (key ? qd.K : qd.V) + code_row<FMT>(pg, qd, id, head, at) + c * code_bits<FMT>() / 8;
    const float s = scale_of(((key ? qd.Ks : qd.Vs) + scale_row(pg, qd, id, head, at))[c / Q_BLOCK]);
    uint32_t w[2];
    if constexpr (FMT == GRACEKV_E4M3) {
      const uint2 u = *(const uint2*)codes;
      w[0] = u.x; w[1] = u.y;
    } else {
      w[0] = *(const uint32_t*)codes;
    }
    x = eight_bf16<FMT>(w, s);
  }
  if constexpr (sizeof(T) == 2) {
    *(uint4*)(dst + c) = x;
  } else {
    float f[8];
    Eight<uint16_t>{x}.get(f);
    Eight<float>::put(dst + c, f);
  }
}

hipError_t launch_quant_append(const PageDims& pg, int format, const QuantDims& qd, const AppendDims& ap, const void* k, const void* v,
                               const void* q, const int32_t* table, const int32_t* start, const int32_t* cu, const int32_t* pos,
                               const float* cosT, const float* sinT, void* q_out, hipStream_t st) {
  if (ap.n_new == 0) return hipSuccess;
  by_type(pg, format, [&](auto type, auto dim, auto fmt) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, FMT = decltype(fmt)::value;
    const int units = (2 * pg.G + (q ? pg.H : 0)) * (D / 16);
    hipLaunchKernelGGL((k_quant_append<T, D, FMT>), dim3((unsigned)ap.n_new, (unsigned)((units + QC_T - 1) / QC_T)), dim3(QC_T), 0, st,
                       pg, qd, ap, (const T*)k, (const T*)v, (const T*)q, table, start, cu, pos, cosT, sinT, (T*)q_out);
  });
  return hipGetLastError();
}

hipError_t launch_quant_read(const PageDims& pg, int format, const QuantDims& qd, const ReadDims& rd, const int32_t* table,
                             const int32_t* start, const int32_t* cu, void* k, void* v, hipStream_t st) {
  if (rd.n_rows == 0) return hipSuccess;
  by_type(pg, format, [&](auto type, auto dim, auto fmt) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, FMT = decltype(fmt)::value;
    const int units = 2 * pg.G * (D / 8);
    hipLaunchKernelGGL((k_quant_read<T, D, FMT>), dim3((unsigned)rd.n_rows, (unsigned)((units + QC_T - 1) / QC_T)), dim3(QC_T), 0, st,
                       pg, qd, rd, table, start, cu, (T*)k, (T*)v);
  });
  return hipGetLastError();
}

}  // namespace gkv
