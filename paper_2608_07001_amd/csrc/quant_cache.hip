// New tokens into a quantised paged cache, keys rotated to their position on the way, and rows
// of it back.
//
//   K[place] <- Q(R(pos) k),  V[place] <- Q(v),  q_out <- R(pos) q      (quant.h for Q)
//   R(p): (x_i, x_{i + d/2}) -> (x_i c - x_{i+d/2} s, x_{i+d/2} c + x_i s), row p of the tables
//   k[row] <- what K[place] stands for,  v[row] likewise
//
// A rotated key is quantised from fp32, where its two products and their sum are each rounded
// (no fused multiply and add: the same codes wherever the rotation is formed like that), and
// not rounded to the rows' type before.  Reading back is exact in fp32, and in bf16 wherever bf16 holds the value.
#include <algorithm>

#include "quant.h"

namespace gkv {

constexpr int QC_T = 256;
typedef int i32x4 __attribute__((ext_vector_type(4)));

// 16 bytes that pass by the caches, through which the chip writes slower: 32K tokens of the 8B heads read back 41 us, 61
// through them; a fill reaches 6.9 TB/s, a copy through them 5.1.  What reads the rows next loses less than that
// (us with the reader behind, past and through; 32 query heads): 12300 rows read back and 300 queries over them 104, 104; 32256 and 256
// 187, 185; 4160 and 64 32.7, 34.4; a prompt of 2048 appended, read back and attended to 75.1, 74.7, of 8192 550, 556; a step of 1,
// 64 and 256 tokens appended and attended to 13.0, 29.3, 39.5 either way.
__device__ __forceinline__ void put_past(void* p, uint4 x) { __builtin_nontemporal_store(__builtin_bit_cast(i32x4, x), (i32x4*)p); }

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
    put_past(p, make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])));
  }
};
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) { a = *(const float4*)p; b = *(const float4*)(p + 4); }
  __device__ __forceinline__ void get(float* x) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  static __device__ __forceinline__ void put(float* p, const float* x) {
    put_past(p, __builtin_bit_cast(uint4, make_float4(x[0], x[1], x[2], x[3])));
    put_past(p + 4, __builtin_bit_cast(uint4, make_float4(x[4], x[5], x[6], x[7])));
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

// Rows of a workgroup: the page and the place in it of each, page -1 where there is none or
// the row is in no sequence (`in`: it is in one).
constexpr int QC_ROWS = 16;
struct Places {
  int id[QC_ROWS], at[QC_ROWS];
  bool in[QC_ROWS];
};
// ... of rows t0 .. t0 + rows - 1, by the first wave.  Up to 64 sequences' starts are asked for at once
// and each row's is found among them; of more, one search for the first row and one for the last
// tell what most workgroups need, and only where sequences change in between each lane looks by itself.
__device__ __forceinline__ void find_places(const PageDims& pg, const int32_t* table, const int32_t* start, const int32_t* cu, int64_t n,
                                            int64_t t0, int rows, Places& to) {
  const int lane = threadIdx.x;
  const int64_t t = t0 + lane;
  int b = 0, first = 0;
  Span sp{0, 0};
  if (pg.n_seq <= 64) {
    const int x = min(lane, pg.n_seq - 1);
    const int c0 = cu[x], c1 = cu[x + 1], s = start[x];
    auto last_at = [&](int64_t row) { return max(__popcll(__ballot(lane < pg.n_seq && c0 <= row)) - 1, 0); };      // as find_span has it
    auto take = [&](int at) {
      const int32_t span[2] = {__builtin_amdgcn_readlane(c0, at), __builtin_amdgcn_readlane(c1, at)};
      b = at;
      first = __builtin_amdgcn_readlane(s, at);
      sp = span_of(span, 0, n);
    };
    const int lo = last_at(t0), hi = last_at(t0 + rows - 1);
    take(lo);
    for (int r = 1; r < rows && lo != hi; ++r) {         // a sequence ends among them
      const int at = last_at(t0 + r);
      const int was_b = b, was_first = first;
      const Span was = sp;
      take(at);
      if (lane < r) { b = was_b; first = was_first; sp = was; }
    }
  } else {
    b = find_span(cu, pg.n_seq, t0);
    if (rows > 1 && find_span(cu, pg.n_seq, t0 + rows - 1) != b) b = span_with(cu, pg.n_seq, t0 + min(lane, rows - 1));
    sp = span_of(cu, b, n);
    first = start[b];
  }
  if (lane >= rows) return;
  const bool in = t >= sp.a && t < sp.a + sp.n;
  const int64_t place = (int64_t)first + (t - sp.a);
  int id = -1;
  if (in && place >= 0 && place < ((int64_t)pg.width << pg.shift)) {
    const int x = table[(int64_t)b * pg.width + (place >> pg.shift)];
    id = x >= 0 && x < pg.n_pages ? x : -1;
  }
  to.in[lane] = in;
  to.id[lane] = id;
  to.at[lane] = (int)(place & (((int64_t)1 << pg.shift) - 1));
}

// A workgroup takes `rows` neighbouring tokens: a unit is eight dims of either half of one head, a
// thread has UN of them in flight.  The tokens' rows are asked for before it is known where they go.
template <typename T, int D, int FMT, int UN>
__global__ __launch_bounds__(QC_T) void k_quant_append(PageDims pg, QuantDims qd, AppendDims ap, int rows, const T* __restrict__ k,
                                                       const T* __restrict__ v, const T* q, const int32_t* __restrict__ table,
                                                       const int32_t* __restrict__ start, const int32_t* __restrict__ cu,
                                                       const int32_t* __restrict__ pos, const float* __restrict__ cosT,
                                                       const float* __restrict__ sinT, T* q_out) {
#pragma clang fp contract(off)
  constexpr int U = D / 16;
  __shared__ Places at;
  __shared__ __align__(16) float sC[QC_ROWS][D / 2], sS[QC_ROWS][D / 2];
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * rows;
  rows = (int)min((int64_t)rows, ap.n_new - t0);
  const int each = (2 * pg.G + (q ? pg.H : 0)) * U, units = rows * each;     // slots: K heads, V heads, query heads
  struct Unit {
    int r, slot, c;
  };
  auto unit = [&](int u) {
    Unit x;
    x.r = (uint32_t)u / (uint32_t)each;
    const int w = u - x.r * each;
    x.slot = w / U;
    x.c = (w % U) * 8;
    return x;
  };
  for (int u0 = UN == 1 ? blockIdx.y * QC_T : 0, once = 0; u0 < units && !(UN == 1 && once); u0 += UN * QC_T, once = 1) {
    Eight<T> lo[UN], hi[UN];
    Unit un[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int u = u0 + i * QC_T + tid;
      un[i] = unit(u < units ? u : 0);
      const int s = un[i].slot;
      const int64_t t = t0 + un[i].r;
      const T* src = s < pg.G ? k + t * ap.k_tok + s * ap.k_head
                              : (s < 2 * pg.G ? v + t * ap.v_tok + (s - pg.G) * ap.v_head : q + t * ap.q_tok + (s - 2 * pg.G) * ap.q_head);
      lo[i].load(src + un[i].c);
      hi[i].load(src + un[i].c + D / 2);
    }
    if (!once) {
      if (tid < 64) find_places(pg, table, start, cu, ap.n_new, t0, rows, at);
      if (pos) {                       // the rows' angles, where their position has some, by the last waves first
        for (int i = QC_T - 1 - tid; i < rows * (D / 8); i += QC_T) {
          const int r = i / (D / 8), c = (i % (D / 8)) * 4;
          const int64_t p = pos[t0 + r];
          if (p >= 0 && p < ap.rope_rows) {
            *(float4*)&sC[r][c] = *(const float4*)(cosT + p * (D / 2) + c);
            *(float4*)&sS[r][c] = *(const float4*)(sinT + p * (D / 2) + c);
          }
        }
      }
      sync_after_lds_stores();
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      if (u0 + i * QC_T + tid >= units) break;
      const int r = un[i].r, s = un[i].slot, c = un[i].c;
      const int64_t t = t0 + r;
      const bool key = s < pg.G, value = !key && s < 2 * pg.G;
      if (at.id[r] < 0) continue;
      if (pos) {
        const int64_t p = pos[t];
        if (p < 0 || p >= ap.rope_rows) continue;
      }
      float x[8], y[8];
      lo[i].get(x);
      hi[i].get(y);
      if (pos && !value) {
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const float4 fc = *(const float4*)&sC[r][c + j], fs = *(const float4*)&sS[r][c + j];
          const float cs[4] = {fc.x, fc.y, fc.z, fc.w}, sn[4] = {fs.x, fs.y, fs.z, fs.w};
#pragma unroll
          for (int m = 0; m < 4; ++m) {
            const float a = x[j + m], e = y[j + m];
            x[j + m] = a * cs[m] - e * sn[m];
            y[j + m] = e * cs[m] + a * sn[m];
          }
        }
      }
      if (key || value) {
        const int head = key ? s : s - pg.G;
        uint8_t* codes = (key ? qd.K : qd.V) + code_row<FMT>(pg, qd, at.id[r], head, at.at[r]);
        uint8_t* scales = (key ? qd.Ks : qd.Vs) + scale_row(pg, qd, at.id[r], head, at.at[r]);
        constexpr int B = code_bits<FMT>();
        const bool first = c % Q_BLOCK == 0;
        put_codes<FMT>(x, codes + c * B / 8, scales + c / Q_BLOCK, first);
        put_codes<FMT>(y, codes + (c + D / 2) * B / 8, scales + (c + D / 2) / Q_BLOCK, first);
      } else {
        T* dst = q_out + t * ap.o_tok + (s - 2 * pg.G) * ap.o_head;
        Eight<T>::put(dst + c, x);
        Eight<T>::put(dst + c + D / 2, y);
      }
    }
  }
}

// A workgroup takes `rows` neighbouring rows; a unit is eight dims of one head
template <typename T, int D, int FMT>
__global__ __launch_bounds__(QC_T) void k_quant_read(PageDims pg, QuantDims qd, ReadDims rd, int rows, const int32_t* __restrict__ table,
                                                     const int32_t* __restrict__ start, const int32_t* __restrict__ cu,
                                                     T* __restrict__ k, T* __restrict__ v) {
  constexpr int U = D / 8, UN = 8, W = FMT == GRACEKV_E4M3 ? 2 : 1;
  __shared__ Places at;
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * rows;
  rows = (int)min((int64_t)rows, rd.n_rows - t0);
  const int sides = (k ? 1 : 0) + (v ? 1 : 0), each = sides * pg.G * U, units = rows * each;
  if (tid < 64) find_places(pg, table, start, cu, rd.n_rows, t0, rows, at);
  sync_after_lds_stores();
  for (int u0 = 0; u0 < units; u0 += UN * QC_T) {
    uint32_t w[UN][W];
    float sc[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int u = u0 + i * QC_T + tid;
      sc[i] = 0.f;
#pragma unroll
      for (int j = 0; j < W; ++j) w[i][j] = 0;               // no page: nothing is there
      if (u >= units) continue;
      const int r = (uint32_t)u / (uint32_t)each, x = u - r * each, s = x / U, c = (x % U) * 8;
      if (at.id[r] < 0) continue;
      const bool key = k && s < pg.G;
      const int head = s < pg.G ? s : s - pg.G;
      const uint8_t* codes = (key ? qd.K : qd.V) + code_row<FMT>(pg, qd, at.id[r], head, at.at[r]) + c * code_bits<FMT>() / 8;
      sc[i] = scale_of(((key ? qd.Ks : qd.Vs) + scale_row(pg, qd, at.id[r], head, at.at[r]))[c / Q_BLOCK]);
      if constexpr (W == 2) {
        const uint2 y = *(const uint2*)codes;
        w[i][0] = y.x; w[i][1] = y.y;
      } else {
        w[i][0] = *(const uint32_t*)codes;
      }
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int u = u0 + i * QC_T + tid;
      if (u >= units) break;
      const int r = (uint32_t)u / (uint32_t)each, x = u - r * each, s = x / U, c = (x % U) * 8;
      if (!at.in[r]) continue;
      const bool key = k && s < pg.G;
      const int head = s < pg.G ? s : s - pg.G;
      T* dst = (key ? k + (t0 + r) * rd.k_tok + head * rd.k_head : v + (t0 + r) * rd.v_tok + head * rd.v_head) + c;
      if constexpr (sizeof(T) == 2) {
        put_past(dst, eight_bf16<FMT>(w[i], sc[i]));
      } else {
        float f[8];
        eight_f32<FMT>(w[i], sc[i], f);
        Eight<float>::put(dst, f);
      }
    }
  }
}

// rows of a workgroup: as many as its threads have in flight, while the chip is full
static int rows_of_group(int64_t n, int units_of_row, int in_flight) {
  const int64_t fit = std::max(1, in_flight * QC_T / units_of_row), full = std::max<int64_t>(1, n / 1024);
  return (int)std::min<int64_t>({fit, full, QC_ROWS});
}

hipError_t launch_quant_append(const PageDims& pg, int format, const QuantDims& qd, const AppendDims& ap, const void* k, const void* v,
                               const void* q, const int32_t* table, const int32_t* start, const int32_t* cu, const int32_t* pos,
                               const float* cosT, const float* sinT, void* q_out, hipStream_t st) {
  if (ap.n_new == 0) return hipSuccess;
  by_type(pg, format, [&](auto type, auto dim, auto fmt) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, FMT = decltype(fmt)::value;
    const int each = (2 * pg.G + (q ? pg.H : 0)) * (D / 16);
    auto run = [&](auto un, dim3 grid, int rows) {
      hipLaunchKernelGGL((k_quant_append<T, D, FMT, decltype(un)::value>), grid, dim3(QC_T), 0, st, pg, qd, ap, rows, (const T*)k,
                         (const T*)v, (const T*)q, table, start, cu, pos, cosT, sinT, (T*)q_out);
    };
    // units in flight of a thread: prompts of 8192 and 2047 tokens, bf16, 62.3 us with 2, 61.3 with 4, 68.9 with 8; of an
    // fp32 unit, twice as long, 2.  Below 1024 tokens every unit has a thread: 64 of a token each 6.2 us
    constexpr int UN = sizeof(T) == 2 ? 4 : 2;
    const int rows = rows_of_group(ap.n_new, each, UN);
    if (ap.n_new < 1024) run(std::integral_constant<int, 1>{}, dim3((unsigned)ap.n_new, (unsigned)((each + QC_T - 1) / QC_T)), 1);
    else run(std::integral_constant<int, UN>{}, dim3((unsigned)((ap.n_new + rows - 1) / rows)), rows);
  });
  return hipGetLastError();
}

hipError_t launch_quant_read(const PageDims& pg, int format, const QuantDims& qd, const ReadDims& rd, const int32_t* table,
                             const int32_t* start, const int32_t* cu, void* k, void* v, hipStream_t st) {
  if (rd.n_rows == 0) return hipSuccess;
  by_type(pg, format, [&](auto type, auto dim, auto fmt) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, FMT = decltype(fmt)::value;
    const int rows = rows_of_group(rd.n_rows, ((k != nullptr) + (v != nullptr)) * pg.G * (D / 8), 8);
    hipLaunchKernelGGL((k_quant_read<T, D, FMT>), dim3((unsigned)((rd.n_rows + rows - 1) / rows)), dim3(QC_T), 0, st,
                       pg, qd, rd, rows, table, start, cu, (T*)k, (T*)v);
  });
  return hipGetLastError();
}

}  // namespace gkv
