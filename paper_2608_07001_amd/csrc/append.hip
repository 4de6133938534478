// New tokens into a paged cache: keys rotated to their position, values as they are,
// both into the sequences' pages, and the tokens' queries rotated in the same launch.
//
//   K[page][g][at] <- R(pos) k,   V[page][g][at] <- v,   q_out <- R(pos) q
//   R(p): (x_i, x_{i + d/2}) -> (x_i c - x_{i+d/2} s, x_{i+d/2} c + x_i s), row p of the tables
//
// Token i of sequence b goes to place start[b] + i of that sequence; a place that its
// row of the block table does not name (past its end, or an id that is no page) and a
// position outside the tables leave the token out.
//
// Everything is read once and written once: the bound is memory, and for one token of
// each sequence the chain sequence -> page -> row.  A lane turns eight pairs (16 bytes
// of either half; fp32: four), rounding once, and the lanes of a head are neighbours; a
// workgroup belongs to one token, so the chain is walked once for all its heads.
// Measured: 10239 tokens of the 8B heads 51 us, 257 MB at 5.0 TB/s (a copy reaches 4.9);
// one token of 64 sequences 2.8 us.
#include "common.h"
#include "pages.h"
#include "serve.h"

namespace gkv {

constexpr int AP_T = 256;

// one 16-byte chunk of either half of a row, as floats
template <typename T> struct Half;
template <> struct Half<uint16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(uint4 u, float* x) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
  }
};
template <> struct Half<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(uint4 u, float* x) {
    x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float* x) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  }
};

template <typename T, int D>
__global__ __launch_bounds__(AP_T) void k_append(PageDims pg, AppendDims ap, const T* __restrict__ k,
                                                 const T* __restrict__ v, const T* q, const int32_t* __restrict__ table,
                                                 const int32_t* __restrict__ start, const int32_t* __restrict__ cu,
                                                 const int32_t* __restrict__ pos, const float* __restrict__ cosT,
                                                 const float* __restrict__ sinT, T* __restrict__ Kp, T* __restrict__ Vp,
                                                 T* q_out) {
  constexpr int N = Half<T>::N, U = D / 2 / N;         // lanes of a head
  const int64_t t = blockIdx.x;
  const int unit = blockIdx.y * AP_T + threadIdx.x;
  const int slot = unit / U, c = (unit % U) * N;       // slot: K heads, V heads, query heads
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
  const T* src;
  T* dst;
  bool turn = pos != nullptr;
  if (slot < pg.G) {
    src = k + t * ap.k_tok + slot * ap.k_head;
    dst = Kp + page_row(pg, id, slot, at);
  } else if (slot < 2 * pg.G) {
    src = v + t * ap.v_tok + (slot - pg.G) * ap.v_head;
    dst = Vp + page_row(pg, id, slot - pg.G, at);
    turn = false;
  } else {
    src = q + t * ap.q_tok + (slot - 2 * pg.G) * ap.q_head;
    dst = q_out + t * ap.o_tok + (slot - 2 * pg.G) * ap.o_head;
  }
  uint4 lo = *(const uint4*)(src + c), hi = *(const uint4*)(src + c + D / 2);
  if (turn) {
    float x[N], y[N], cs[N], sn[N], a[N], e[N];
    Half<T>::get(lo, x);
    Half<T>::get(hi, y);
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const float4 fc = *(const float4*)(cosT + p * (D / 2) + c + i), fs = *(const float4*)(sinT + p * (D / 2) + c + i);
      cs[i] = fc.x; cs[i + 1] = fc.y; cs[i + 2] = fc.z; cs[i + 3] = fc.w;
      sn[i] = fs.x; sn[i + 1] = fs.y; sn[i + 2] = fs.z; sn[i + 3] = fs.w;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      a[i] = x[i] * cs[i] - y[i] * sn[i];
      e[i] = y[i] * cs[i] + x[i] * sn[i];
    }
    lo = Half<T>::put(a);
    hi = Half<T>::put(e);
  }
  *(uint4*)(dst + c) = lo;
  *(uint4*)(dst + c + D / 2) = hi;
}

hipError_t launch_append(const PageDims& pg, const AppendDims& ap, const void* k, const void* v, const void* q,
                         const int32_t* table, const int32_t* start, const int32_t* cu, const int32_t* pos,
                         const float* cosT, const float* sinT, void* Kp, void* Vp, void* q_out, hipStream_t st) {
  if (ap.n_new == 0) return hipSuccess;
  const int slots = 2 * pg.G + (q ? pg.H : 0);
  auto go = [&](auto type, auto dim) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value;
    const int units = slots * (D / 2 / Half<T>::N);
    hipLaunchKernelGGL((k_append<T, D>), dim3((unsigned)ap.n_new, (unsigned)((units + AP_T - 1) / AP_T)), dim3(AP_T), 0, st, pg,
                       ap, (const T*)k, (const T*)v, (const T*)q, table, start, cu, pos, cosT, sinT, (T*)Kp, (T*)Vp, (T*)q_out);
  };
  if (pg.dtype == GRACEKV_BF16) {
    if (pg.d == 128) go(uint16_t{}, std::integral_constant<int, 128>{}); else go(uint16_t{}, std::integral_constant<int, 64>{});
  } else {
    if (pg.d == 128) go(float{}, std::integral_constant<int, 128>{}); else go(float{}, std::integral_constant<int, 64>{});
  }
  return hipGetLastError();
}

}  // namespace gkv
