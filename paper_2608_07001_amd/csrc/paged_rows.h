// How the rows (sequence, KV head) of attention over pages are cut into chunks on the device,
// and how the states of a chunk's waves, of a row's chunks and of another attention over
// further entries become one result: what the kernels over plain (paged.hip) and quantised
// pages (quant_paged.hip) have in common.
#pragma once

#include "tickets.h"

namespace gkv {

// The last chunk of a row joins PA_JOIN states at a time (32 are up to a fifth slower, 16 the
// same; four dims a lane instead of two joins 16 heads faster, 128K tokens of one KV head 48 us
// instead of 55, and the others slower).
constexpr int PA_JOIN = 8;

// Workspace: a ticket word for every row and group of heads, then per chunk and head
// (max, sum), then the partial sums [chunk][hpg][d].
struct PagedWs {
  unsigned long long* ticket;
  unsigned long long* ml;
  float* o;
  size_t bytes;
};
GKV_HD int ticket_step(const PageDims& pg) { return (int64_t)pg.n_seq * pg.G * ((pg.hpg + PA_HEADS - 1) / PA_HEADS) <= 4096 ? 16 : 1; }
static inline PagedWs paged_view(void* base, const PageDims& pg) {
  const size_t R = (size_t)pg.n_seq * pg.G, chunks = R + PA_TARGET;
  char* p = (char*)base;
  PagedWs w;
  size_t o = 0;
  w.ticket = (unsigned long long*)(p + o);
  o += al256(R * ((pg.hpg + PA_HEADS - 1) / PA_HEADS) * ticket_step(pg) * 8);
  w.ml = (unsigned long long*)(p + o);
  o += al256(chunks * pg.hpg * 8);
  w.o = (float*)(p + o);
  o += chunks * pg.hpg * pg.d * 4;
  w.bytes = o;
  return w;
}

// inclusive sum over the lanes of the wave
__device__ __forceinline__ int scan_wave(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);     // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  const int r = (threadIdx.x & 63) >> 4;
  const int a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31), c = __builtin_amdgcn_readlane(v, 47);
  return v + (r > 0 ? a : 0) + (r > 1 ? b : 0) + (r > 2 ? c : 0);
}

// What a workgroup works on: tiles [t0, t1) of row (b, g); chunk `c` of `chunks`.
struct Chunk {
  int b, g, c, chunks, t0, t1;
};

// The chunk of place `bid` of `places`; false past the last.  Rows are looked at as units:
// (b, g) where a prefix makes their lengths differ, b (G equal rows) otherwise.  Every
// wave finds it by itself, 64 units at a time; over that few it takes one round of loads
// and scans without a barrier.  With more units the waves share a first look at them all,
// which is enough where no row needs a second chunk (4096 sequences of 64 tokens: 860 us
// with the search, 403 without).  W: waves of the workgroup; of eight, no more chunks than run
// at once (one_round).
template <int TILE, bool PREFIX, int W = PA_W>
__device__ __forceinline__ bool find_chunk(const PageDims& pg, const PrefixView& px, const int32_t* len, int bid, int places, float join,
                                           Chunk& out) {
  const int lane = threadIdx.x & 63;
  const int units = PREFIX ? pg.n_seq * pg.G : pg.n_seq, mult = PREFIX ? 1 : pg.G;
  auto tiles = [&](int u) -> int {
    if (u >= units) return 0;
    int64_t s = 0;
    return tiles_of<TILE>(held_len(pg, len[PREFIX ? u / pg.G : u]), PREFIX ? held_count(px, u, s) : 0);
  };
  const int room = places - pg.n_seq * pg.G;
  int first = 0, first_chunks = 0, size;        // of the lane's unit in the first round
  if (units <= 64) {
    first = tiles(lane);
    const uint64_t total = (uint64_t)(uint32_t)__builtin_amdgcn_readlane(scan_wave(first), 63) * mult;
    size = chunk_tiles(total, room);
    if constexpr (W > PA_W) {
      first_chunks = first ? chunks_of(first, size, join) : 0;
      const int fit = one_round(total, pg.n_seq * pg.G, size, (int64_t)__builtin_amdgcn_readlane(scan_wave(first_chunks), 63) * mult);
      if (fit != size) {
        size = fit;
        first_chunks = first ? chunks_of(first, size, join) : 0;
      }
    }
  } else {
    __shared__ uint64_t part[W];
    __shared__ int most[W];
    uint64_t sum = 0;
    int mx = 0;
    for (int u = threadIdx.x; u < units; u += 64 * W) {
      const int n = tiles(u);
      sum += n;
      mx = max(mx, n);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      sum += __shfl_xor(sum, o, 64);
      mx = max(mx, __shfl_xor(mx, o, 64));
    }
    if (lane == 0) { part[threadIdx.x >> 6] = sum; most[threadIdx.x >> 6] = mx; }
    sync_after_lds_stores();
    sum = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) { sum += part[i]; mx = max(mx, most[i]); }
    size = chunk_tiles(sum * mult, room);
    if constexpr (W > PA_W) size = one_round(sum * mult, pg.n_seq * pg.G, size, places);
    size = __builtin_amdgcn_readfirstlane(size);
    if (__builtin_amdgcn_readfirstlane(mx) <= size) {
      if (bid >= units * mult) return false;
      const int u = bid / mult;
      out.b = PREFIX ? u / pg.G : u;
      out.g = PREFIX ? u % pg.G : bid % mult;
      out.c = 0;
      out.chunks = 1;
      out.t0 = 0;
      out.t1 = __builtin_amdgcn_readfirstlane(tiles(u));
      return true;
    }
    first = tiles(lane);
  }
  // the rows of several chunks first, then the others, which even out the end (where there
  // are more units than a wave looks at in one round, rows as they come: their end is short)
  const bool ordered = units <= 64;
  int base = 0;
#pragma unroll 1
  for (int many = 1; many >= (ordered ? 0 : 1); --many)
#pragma unroll 1
    for (int u0 = 0; u0 < units; u0 += 64) {
      const int n = u0 ? tiles(u0 + lane) : first, x = W > PA_W && ordered ? first_chunks : n ? chunks_of(n, size, join) : 0;
      const int c = !ordered || (x > 1) == many ? x * mult : 0;
      const int to = scan_wave(c);     // at most the places: no overflow
      const int all = base + __builtin_amdgcn_readlane(to, 63);
      if (bid < all) {
        const int at = __popcll(__ballot(base + to <= bid));       // the unit's lane
        const int u = u0 + at;
        const int tn = __builtin_amdgcn_readlane(n, at), chunks = __builtin_amdgcn_readlane(x, at);
        const int local = bid - base - (__builtin_amdgcn_readlane(to, at) - chunks * mult);
        out.b = PREFIX ? u / pg.G : u;
        out.g = PREFIX ? u % pg.G : local / chunks;
        out.c = PREFIX ? local : local % chunks;
        out.chunks = chunks;
        const int each = tn / chunks, more = tn % chunks;            // the first `more` take one more
        out.t0 = out.c * each + min(out.c, more);
        out.t1 = out.t0 + each + (out.c < more);
        return true;
      }
      base = all;
    }
  return false;
}

// What the waves of a workgroup have of chunk `ck` (sM, sL, sO: maximum, sum and weighted
// values of every wave and head; written, with a barrier behind): merged, written as the row's
// result where the chunk is all of it, else left in the workspace, for the last of the row's
// chunks to join.  `part` (o not null): an attention of the same queries over other entries,
// joined to the row's as a state of its own, maximum lse, sum 1 and its mean.
template <typename T, int D, bool RAISED, int JOIN, int W = PA_W>
__device__ __forceinline__ void finish_row(const PageDims& pg, const Chunk& ck, const PagedWs& ws, const PartView& part, int bid,
                                           int group, int groups, const float (*sM)[PA_HEADS], const float (*sL)[PA_HEADS],
                                           const float (*sO)[PA_HEADS][D + 4], T* __restrict__ out, float* __restrict__ lse) {
  __shared__ int joins;
  constexpr float LOG2E = 1.44269504088896341f;
  const int tid = threadIdx.x;
  const int h0 = group * PA_HEADS, heads = min(PA_HEADS, pg.hpg - h0);
  const int64_t row = (int64_t)ck.b * pg.G + ck.g;
  // state (m, s, o) onto (M, S, O): one of no entry has the maximum -inf and adds nothing,
  // unless its sum is no number
  auto add = [&](float& M, float& S, float& O0, float& O1, float m2, float s2, float a0, float a1) {
    const float mn = fmaxf(M, m2);
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((M - mn) * LOG2E);
    const float c = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m2 - mn) * LOG2E);
    S = (f == 0.f && S == S ? 0.f : S * f) + (c == 0.f && s2 == s2 ? 0.f : s2 * c);
    O0 = (f == 0.f ? 0.f : O0 * f) + (c == 0.f ? 0.f : a0 * c);
    O1 = (f == 0.f ? 0.f : O1 * f) + (c == 0.f ? 0.f : a1 * c);
    M = mn;
  };
  auto finish = [&](int h, int dd, float M, float S, float O0, float O1) {
    const int64_t hd = (int64_t)ck.b * pg.H + (int64_t)ck.g * pg.hpg + h0 + h;
    if (part.o) {
      const float2 x = *(const float2*)(part.o + hd * D + dd);
      add(M, S, O0, O1, part.lse[hd], 1.f, x.x, x.y);
    }
    stf(out, hd * D + dd, S > 0.f ? O0 / S : S);                  // nothing: 0; NaN stays
    stf(out, hd * D + dd + 1, S > 0.f ? O1 / S : S);
    if (lse && dd == 0) lse[hd] = M + logf(S);
  };
  const int64_t place = (int64_t)bid * pg.hpg + h0;
  for (int i = tid; i < heads * (D / 2); i += 64 * W) {
    const int h = i / (D / 2), dd = 2 * (i % (D / 2));
    float M = -INFINITY, S = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
    for (int x = 0; x < W; ++x) add(M, S, O0, O1, sM[x][h], sL[x][h], sO[x][h][dd], sO[x][h][dd + 1]);
    if (ck.chunks == 1) {
      finish(h, dd, M, S, O0, O1);
    } else {
      put_agent((unsigned long long*)(ws.o + (place + h) * D + dd), pair_bits(O0, O1));
      if (dd == 0) put_agent(ws.ml + place + h, pair_bits(M, S));
    }
  }
  if (ck.chunks == 1) return;
  stores_done();
  __syncthreads();
  if (tid == 0) joins = last_of<RAISED>(ws.ticket + (row * groups + group) * ticket_step(pg), ck.chunks);
  sync_after_lds_stores();
  if (!joins) return;
  // A head's pairs of dims lie on LH neighbouring lanes, which hold the (max, sum) of LH
  // chunks at a time, one each, and pass the weights round.
  constexpr int LH = D / 2;
  const int64_t base = (int64_t)(bid - ck.c) * pg.hpg + h0;              // the row's first chunk
  for (int i = tid; i < (heads * LH + 63) / 64 * 64; i += 64 * W) {               // whole waves
    const int h = min(i / LH, heads - 1), sub = i % LH, dd = 2 * sub;
    float M = -INFINITY, S = 0.f, O0 = 0.f, O1 = 0.f;
    for (int b0 = 0; b0 < ck.chunks; b0 += LH) {
      const int nb = min(ck.chunks - b0, LH);
      const unsigned long long* src = (const unsigned long long*)(ws.o + (base + (int64_t)b0 * pg.hpg + h) * D + dd);
      const int64_t step = (int64_t)pg.hpg * LH;
      unsigned long long ov[JOIN];
      auto load = [&](int c0) {                 // past the last: that one again
#pragma unroll
        for (int c = 0; c < JOIN; ++c) ov[c] = ld_agent(src + min(c0 + c, nb - 1) * step);
      };
      float2 ml = make_float2(-INFINITY, 0.f);
      if (sub < nb) ml = pair_of(ld_agent(ws.ml + base + (int64_t)(b0 + sub) * pg.hpg + h));
      load(0);
      float mb = ml.x;
#pragma unroll
      for (int o = LH / 2; o > 0; o >>= 1) mb = fmaxf(mb, __shfl_xor(mb, o, 64));
      const float f = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((ml.x - mb) * LOG2E);
      float sb = f == 0.f && ml.y == ml.y ? 0.f : ml.y * f;                     // NaN stays
#pragma unroll
      for (int o = LH / 2; o > 0; o >>= 1) sb += __shfl_xor(sb, o, 64);
      float a0 = 0.f, a1 = 0.f;
      for (int c0 = 0; c0 < nb; c0 += JOIN) {
        if (c0) load(c0);
#pragma unroll
        for (int c = 0; c < JOIN; ++c) {
          const float g = c0 + c < nb ? __shfl(f, (tid & 63 & ~(LH - 1)) + c0 + c, 64) : 0.f;
          const float2 v = pair_of(ov[c]);
          a0 += g == 0.f ? 0.f : v.x * g;
          a1 += g == 0.f ? 0.f : v.y * g;
        }
      }
      add(M, S, O0, O1, mb, sb, a0, a1);
    }
    if (i < heads * LH) finish(h, dd, M, S, O0, O1);
  }
}

}  // namespace gkv
