// Attention of one new token of every sequence over its pages of quantised keys and values
// (quant.h), and over further entries whose attention is given as a part.
//
// For sequence b and query head h (KV head g = h / hpg) the entries are the first len[b] tokens of
// its pages: out = sum e^x v / sum e^x with x = q.k / sqrt(d), lse = log sum e^x; a part's mean
// and lse are joined to that.  No entry: 0 and -inf.
//
// The work is a stream over codes, each read once for all query heads of its group: bound by
// HBM, d + d / 32 bytes of a row of e4m3 and d / 2 + d / 32 of e2m1.  Rows are cut into chunks, found and
// joined as those of plain pages are (paged_rows.h).
//
// A wave takes tiles of 32 entries.  Codes become bf16 in registers, two a conversion, the
// block's power of two in the same instruction, exactly, and everything goes through the bf16 matrix
// instructions: S^T = K Q^T (entries x heads), whose accumulator holds four entries of one
// head a lane, the operand layout of O^T = V^T P^T.  Which dims a lane has of a key is
// free as long as the query agrees, so a key's codes are loaded 16 bytes a lane; which entry is which row
// of a product is free as well, and is chosen so that a load of values is one piece of memory.
// (The matrix instructions that take codes and scales themselves were measured first: they keep about 14 bits
// below the largest of the products that they add at a time, which a logit's error shows, and a query
// would have to be given to them in 8 bits.)
// bf16 rows: weights in two bf16 parts, off by at most 2^-15 of themselves; fp32 rows: queries and
// weights in three, which is all their bits.
//
// Measured, bf16: 64 sequences of 1 to 8192 tokens, 8 KV heads of 128, 32 query heads, e4m3: 44 us (4.0 TB/s; the
// loads alone take 42: pages of 16 tokens lie 2 KB a head apart); 4 sequences of about 128K, 64 query heads,
// e2m1: 108 us (4.9 TB/s; the loads alone 104), rising to 120 to 140 where such calls follow one another for
// milliseconds; one sequence of 8201 tokens
// 13.1 us, bound by latency: finding the chunk, page ids, the tiles of a wave, the states and their join, one
// after the other.  Two tiles of loads in flight were slower everywhere (15.6, 50.7 and 127 us where one tile
// in flight took 14.6, 44 and 126): their registers leave a wave less a SIMD.
#include <algorithm>

#include "paged_rows.h"
#include "quant.h"

namespace gkv {

constexpr int QP_JOIN = 8;         // states joined at a time: one sequence 13.9 us with 4, 13.1 with 8, 13.4 with 16
constexpr float LAG = 8.f;         // (below) a weight is 2^-8 at the row's largest at the least

// Waves a SIMD that the registers have to leave room for, workgroups of four waves.  With four a SIMD everything spills: 64 sequences
// 106 us for 44.  e4m3 keys beside an fp32 query's three parts do not fit three either: 64 sequences of 4096 tokens,
// 8 KV heads of 128, 32 query heads 171 us with three and 114 with two; of e2m1 80 and 87.
template <typename T, int D, int FMT> constexpr int quant_waves() {
  return sizeof(T) == 4 && D == 128 && FMT == GRACEKV_E4M3 ? 2 : 3;
}

// the value of one lane of the quad
template <int CTRL> __device__ __forceinline__ float quad_of(float x) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, true));
}

template <typename T, int D, int FMT, int W>
__global__ __launch_bounds__(64 * W, (W == 8 ? 2 : quant_waves<T, D, FMT>())) void k_quant_paged(
    PageDims pg, QuantDims qd, int64_t q_tok, const T* __restrict__ q, const int32_t* __restrict__ table, const int32_t* __restrict__ len,
    PartView part, T* __restrict__ out, float* __restrict__ lse, PagedWs ws) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int NS = 2, TILE = 16 * NS, PAIR = W / PA_W;        // (chunks of eight waves are counted in pairs of tiles)
  constexpr int BITS = code_bits<FMT>();
  constexpr int QP = BF ? 1 : 3, PP = BF ? 2 : 3;        // bf16 parts of a query, of a weight
  constexpr int PB = D * BITS / 32 < 16 ? D * BITS / 32 : 16;      // bytes of a lane's piece of a key
  constexpr int KP = D * BITS / 32 / PB;                 // pieces of a lane
  constexpr int PD = PB * 8 / BITS;                      // dims of a piece
  constexpr int KS = D / 32;                             // products over the dims
  constexpr int VD = D / 16;                             // neighbouring dims of a lane in a value row
  constexpr int VB = VD * BITS / 8;                      // ... bytes: 8, 4 or 2
  constexpr int VW = VB < 4 ? 1 : VB / 4;
  constexpr int RB = D * BITS / 8, SB = D / Q_BLOCK;     // bytes of a row and of its scales
  __shared__ float sM[W][PA_HEADS], sL[W][PA_HEADS];
  __shared__ __align__(16) float sO[W][PA_HEADS][D + 4];      // rows start in other banks
  const int groups = (pg.hpg + PA_HEADS - 1) / PA_HEADS;
  const int bid = groups > 1 ? blockIdx.x / groups : blockIdx.x, group = groups > 1 ? blockIdx.x % groups : 0;
  Chunk ck;
  const int places = groups > 1 ? gridDim.x / groups : gridDim.x;
  if (!find_chunk<TILE * PAIR, false, W>(pg, PrefixView{}, len, bid, places, join_cost(pg.hpg, D) / PAIR, ck)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g4 = lane >> 4;
  const int h0 = group * PA_HEADS, heads = min(PA_HEADS, pg.hpg - h0);
  constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
  const float scale = 1.0f / sqrtf((float)D), sc2 = scale * LOG2E;
  const int seq = ck.b, kv = ck.g;
  const int64_t n_page = held_len(pg, len[seq]);
  // the lane's dims of product s: the eight from 4 PD (s / (PD / 8)) + PD g4 + 8 (s % (PD / 8)) on
  uint4 qv[QP][KS];
#pragma unroll
  for (int s = 0; s < KS; ++s) {
    constexpr int PS = PD / 8;
    const T* p = q + seq * q_tok + ((int64_t)kv * pg.hpg + h0 + i16) * D + 4 * PD * (s / PS) + PD * g4 + 8 * (s % PS);
    if constexpr (BF) {
      qv[0][s] = i16 < heads ? *(const uint4*)p : make_uint4(0, 0, 0, 0);
    } else {
      float x[8];
      const float4 a = i16 < heads ? *(const float4*)p : make_float4(0, 0, 0, 0);
      const float4 b = i16 < heads ? *(const float4*)(p + 4) : make_float4(0, 0, 0, 0);
      x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
#pragma unroll
      for (int y = 0; y < QP; ++y) {
        qv[y][s] = make_uint4(uppers(x[0], x[1]), uppers(x[2], x[3]), uppers(x[4], x[5]), uppers(x[6], x[7]));
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] -= upper(x[i]);
      }
    }
  }

  // One tile's codes and scales.  Row j of a product's 16 is entry j / 4 + 4 (j % 4) of a half, so that the
  // lanes of the four value rows r of a lane, entries g4 + 4 r, lie side by side: a load of values is one
  // piece of memory, not four.  A quad of lanes has the scales of its lane group's four rows, one each.
  uint32_t tk[NS][KP][PB / 4], tv[NS][4][VW];
  uint32_t sk[NS], sv[NS];
  struct Where {                  // of a tile, the same for the wave: bytes, entries there are
    int64_t at[NS], sc[NS];
    int n[NS];
  };
  // The page ids of a tile are asked for a tile earlier still: they would stand in front of its loads
  const int32_t* tab = table + (int64_t)seq * pg.width;
  struct Ids {
    int id[NS];
  };
  auto pages_of = [&](int ti) __attribute__((always_inline)) {
    Ids r;
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      const int64_t e = (int64_t)ti * TILE + 16 * h;
      r.id[h] = e < n_page ? tab[e >> pg.shift] : -1;
    }
    return r;
  };
  auto where = [&](int ti, const Ids& ids) __attribute__((always_inline)) {
    Where r;
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      const int64_t e = (int64_t)ti * TILE + 16 * h;
      int64_t left = n_page - e;
      r.at[h] = r.sc[h] = 0;
      const int64_t id = ids.id[h];
      if (id < 0 || id >= pg.n_pages) {
        left = 0;
      } else {
        const int at = (int)(e & (((int64_t)1 << pg.shift) - 1));
        r.at[h] = code_row<FMT>(pg, qd, id, kv, at);
        r.sc[h] = scale_row(pg, qd, id, kv, at);
      }
      r.n[h] = left > 16 ? 16 : (left < 0 ? 0 : (int)left);
    }
    return r;
  };
  const int row_j = (i16 >> 2) + 4 * (i16 & 3), row_s = g4 + 4 * (i16 & 3);
  // a page holds all 16 rows, written or not
  auto load_keys = [&](const Where& t) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      sk[h] = 0;
#pragma unroll
      for (int p = 0; p < KP; ++p)
#pragma unroll
        for (int x = 0; x < PB / 4; ++x) tk[h][p][x] = 0;
      if (t.n[h] == 0) continue;
      const uint8_t* base = qd.K + t.at[h];
#pragma unroll
      for (int p = 0; p < KP; ++p) __builtin_memcpy(tk[h][p], __builtin_assume_aligned(base + (row_j * RB + PB * g4) + 4 * PB * p, PB), PB);
      const uint8_t* s = qd.Ks + t.sc[h] + SB * row_j;
      sk[h] = SB == 4 ? *(const uint32_t*)s : *(const uint16_t*)s;
    }
  };
  auto load_values = [&](const Where& t) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < NS; ++h) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int x = 0; x < VW; ++x) tv[h][r][x] = 0;
      sv[h] = 0;
      if (t.n[h] == 0) continue;
      const uint8_t* base = qd.V + t.at[h];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const uint8_t* x = base + ((g4 + 4 * r) * RB + VB * i16);
        if constexpr (VB == 8) __builtin_memcpy(tv[h][r], __builtin_assume_aligned(x, 8), 8);
        else if constexpr (VB == 4) tv[h][r][0] = *(const uint32_t*)x;
        else tv[h][r][0] = *(const uint16_t*)x;
      }
      const uint8_t* s = qd.Vs + t.sc[h] + SB * row_s;
      sv[h] = SB == 4 ? *(const uint32_t*)s : *(const uint16_t*)s;
    }
  };

  f32x4 o[VD];
#pragma unroll
  for (int j = 0; j < VD; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;               // of head i16; l: this lane's entries only

  const int t1 = min(ck.t1 * PAIR, (int)((n_page + TILE - 1) / TILE));
  int ti = ck.t0 * PAIR + w;
  Where now{}, next{};
  Ids ids{};
  if (ti < t1) {
    now = where(ti, pages_of(ti));
    ids = pages_of(min(ti + W, t1 - 1));
    load_keys(now);
    load_values(now);
  }
  for (; ti < t1; ti += W) {
    const bool more = ti + W < t1;
    if (more) {
      next = where(ti + W, ids);
      ids = pages_of(min(ti + 2 * W, t1 - 1));
    }
    float x[NS][4];
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s) {
        constexpr int PS = PD / 8, W8 = BITS / 4;            // eight values' words
        // the piece lies in one block: that of its first dim
        const uint32_t blk = (uint32_t)(4 * PD * (s / PS) + PD * g4) / Q_BLOCK;
        const float f = scale_of((sk[h] >> (8 * blk)) & 255u);
        const s16x8 k8 = pk8(eight_bf16<FMT>(&tk[h][s / PS][(s % PS) * W8], f));
#pragma unroll
        for (int y = QP - 1; y >= 0; --y) acc = mfma_bf16_16x16x32(k8, pk8(qv[y][s]), acc);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) x[h][r] = BF ? acc[r] : acc[r] * scale;
    }
    if (more) load_keys(next);
    bool all = true;
#pragma unroll
    for (int h = 0; h < NS; ++h) all &= now.n[h] == 16;
    if (!all) {                   // absent entries: no weight, and values that are 0 whatever they hold
#pragma unroll
      for (int h = 0; h < NS; ++h) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool none = g4 + 4 * r >= now.n[h];
          x[h][r] = none ? -INFINITY : x[h][r];
#pragma unroll
          for (int i = 0; i < VW; ++i) tv[h][r][i] = none ? 0 : tv[h][r][i];
        }
        sv[h] = row_s >= now.n[h] ? 0 : sv[h];
      }
    }
    float mx = x[0][0];
#pragma unroll
    for (int h = 0; h < NS; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[h][r]);
    {
      const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
      const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
    }
    // bf16 rows: base-2 units from here, formed with the exponent's argument in one step, and what is
    // subtracted stands LAG above a maximum that may lag behind by as much, so that sums are
    // rescaled seldom (no weight is above 1, the row's largest at least 2^-LAG)
    if constexpr (BF) mx *= sc2;
    if (__any(mx > m)) {
      const float mn = BF ? fmaxf(m, mx + LAG) : fmaxf(m, mx);
      const float c = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(BF ? m - mn : (m - mn) * LOG2E);
      m = mn;
      l *= c;
#pragma unroll
      for (int j = 0; j < VD; ++j) o[j] *= c;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    uint4 pb[PP];                 // the tile's weights, in parts
    {
      float pr[NS][4];
#pragma unroll
      for (int h = 0; h < NS; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if constexpr (BF) {
            pr[h][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[h][r], sc2, -ms));
          } else {
            const float y = (x[h][r] - ms) * LOG2E;
            pr[h][r] = __builtin_amdgcn_exp2f(y);
            // what the product lost, to first order
            if (pr[h][r] > 0.f) pr[h][r] = __builtin_fmaf(pr[h][r], __builtin_fmaf(x[h][r] - ms, LOG2E, -y) * LN2, pr[h][r]);
          }
          l += pr[h][r];
        }
#pragma unroll
      for (int y = 0; y < PP; ++y) {
        if (y == PP - 1) {        // the last: rounded
          pb[y] = make_uint4(pack_bf16(pr[0][0], pr[0][1]), pack_bf16(pr[0][2], pr[0][3]), pack_bf16(pr[1][0], pr[1][1]), pack_bf16(pr[1][2], pr[1][3]));
        } else {
          pb[y] = make_uint4(uppers(pr[0][0], pr[0][1]), uppers(pr[0][2], pr[0][3]), uppers(pr[1][0], pr[1][1]), uppers(pr[1][2], pr[1][3]));
#pragma unroll
          for (int h = 0; h < NS; ++h)
#pragma unroll
            for (int r = 0; r < 4; ++r) pr[h][r] -= upper(pr[h][r]);
        }
      }
    }
    // values of the lane's eight rows as bf16 pairs of neighbouring dims
    uint32_t vv[NS][4][VD / 2];
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      // a quad's lanes have dims of one block
      const float own = scale_of((sv[h] >> (8 * (uint32_t)(VD * i16 / Q_BLOCK))) & 255u);
      float f[4];
      f[0] = quad_of<0x00>(own);
      f[1] = quad_of<0x55>(own);
      f[2] = quad_of<0xAA>(own);
      f[3] = quad_of<0xFF>(own);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        if constexpr (VD == 8) {
          const uint4 u = eight_bf16<FMT>(tv[h][r], f[r]);
          vv[h][r][0] = u.x; vv[h][r][1] = u.y; vv[h][r][2] = u.z; vv[h][r][3] = u.w;
        } else {
          vv[h][r][0] = pair_bf16<FMT, 0>(tv[h][r][0], f[r]);
          vv[h][r][1] = pair_bf16<FMT, 1>(tv[h][r][0], f[r]);
        }
      }
    }
    if (more) load_values(next);
#pragma unroll
    for (int j = 0; j < VD; ++j) {
      const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
      uint32_t a[NS][2];
#pragma unroll
      for (int h = 0; h < NS; ++h)
#pragma unroll
        for (int r = 0; r < 2; ++r) a[h][r] = __builtin_amdgcn_perm(vv[h][2 * r + 1][j / 2], vv[h][2 * r][j / 2], sel);
      const auto v8 = pk8(make_uint4(a[0][0], a[0][1], a[1][0], a[1][1]));
#pragma unroll
      for (int y = PP - 1; y >= 0; --y) o[j] = mfma_bf16_16x16x32(v8, pk8(pb[y]), o[j]);
    }
    if (more) now = next;
  }
  // the row's ticket word is made ready now, for its chunks to count themselves in one step
  if (ck.chunks > 1 && tid == 0) raise(ws.ticket + (((int64_t)seq * pg.G + kv) * groups + group) * ticket_step(pg));
#pragma unroll
  for (int j = 0; j < VD; ++j) mfma_done(o[j]);
  l = col_sum4(l);
  // row 4 g4 + r of product j is dimension VD (4 g4 + r) + j, column i16 the head
  if (g4 == 0) { sM[w][i16] = BF ? m * LN2 : m; sL[w][i16] = l; }
  if (i16 < heads) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VD; j += 4)
        *(float4*)&sO[w][i16][VD * (4 * g4 + r) + j] = make_float4(o[j][r], o[j + 1][r], o[j + 2][r], o[j + 3][r]);
  }
  sync_after_lds_stores();
  finish_row<T, D, true, QP_JOIN, W>(pg, ck, ws, part, bid, group, groups, sM, sL, sO, out, lse);
}

hipError_t launch_quant_paged(const PageDims& pg, int format, const QuantDims& qd, int64_t q_tok, const void* q, const int32_t* table,
                              const int32_t* len, const PartView& part, void* out, float* lse, void* ws, hipStream_t st) {
  const PagedWs v = paged_view(ws, pg);
  const int64_t R = (int64_t)pg.n_seq * pg.G;
  const bool eight = eight_waves(pg);
  const int64_t room = eight ? std::min<int64_t>(chunk_room(pg, 0, 64), 256 - R / 2) : chunk_room(pg, 0, 32);
  const dim3 grid((unsigned)((R + room) * ((pg.hpg + PA_HEADS - 1) / PA_HEADS)));
  by_type(pg, format, [&](auto type, auto dim, auto fmt) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, FMT = decltype(fmt)::value;
    auto run = [&](auto waves) {
      constexpr int W = decltype(waves)::value;
      hipLaunchKernelGGL((k_quant_paged<T, D, FMT, W>), grid, dim3(64 * W), 0, st, pg, qd, q_tok, (const T*)q, table, len, part, (T*)out, lse, v);
    };
    if (eight) run(std::integral_constant<int, 8>{}); else run(std::integral_constant<int, 4>{});
  });
  return hipGetLastError();
}

}  // namespace gkv
