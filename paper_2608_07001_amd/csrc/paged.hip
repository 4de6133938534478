// Attention of one new token of every sequence over its pages, and over the packed
// entries of its compressed context in front of them.
//
// For sequence b and query head h (KV head g = h / hpg) the entries are
//   (a) rows [start, start + count) of the packed arrays (b, g), logits q.k / sqrt(d) + log m
//   (b) the first len[b] tokens of its pages, logits q.k / sqrt(d)
// and out = sum e^x v / sum e^x, lse = log sum e^x; no entry: 0 and -inf.
//
// The work is a stream over keys and values, each read once for all query heads of its
// group: bound by HBM.  Sequences differ in length, and how long they are is known on
// the device only, so the split is made there: every row (b, g) is cut into tiles of 16
// or 32 entries, a chunk is so many tiles that the chunks of all rows fill the chip once
// (few rows) or twice, and every workgroup finds its chunk by a scan over the rows'
// lengths.  A row of one chunk is finished by its workgroup; the chunks of a longer one
// leave a partial state each, and the workgroup that comes last joins them, in their order
// (Tickets).  (Joining in a second launch cost 64 ragged sequences 4 us of 81, the smallest
// call 5 of 14; one line of all rows' tiles cut into equal pieces, rows beginning and ending
// anywhere in them, 114 us instead of 81, for a workgroup then has many short rows, one
// after the other, and the loop over them spills.)
//
// Measured (graph of 12 calls over three states): four caches of 128K tokens, 8 KV heads of
// 128, 8 query heads each, 351 to 362 us for 2.01 GB, 5.6 to 5.7 TB/s (a copy moves 4.9, read
// and write together); 64 sequences of 1 to 8192 tokens 73 us, 4.7 TB/s, of which about 11 us
// are the way to the first byte and from the last; 24 compressed contexts of 2048 entries
// a head 47 us; one of 512 entries a head 9.6 us, latency.
//
// A wave takes whole tiles.  Logits are formed transposed, S^T = K Q^T (entries x heads,
// 16x16 matrix tiles, heads past the group's zero), keys straight from memory as the
// product's operand.  A lane then holds four entries of one head, which is the operand
// layout of the second product O^T = V^T P^T: probabilities never cross lanes.  V^T needs
// the same four entries of one dimension; a lane loads those entries' rows (16 bytes
// each) and pairs the halves up in registers, row i of product j being dimension 8 i + j.
// No LDS before the waves are merged, and one tile's registers serve the next (168 at d =
// 128: three waves a SIMD; two tiles in turn took 236, two waves, and were 2 to 4 % slower).
// bf16 probabilities go into the second product as two bf16 parts, off by at most 2^-15 of
// themselves, so what remains is the output's own rounding.  The matrix pipes wait for memory
// in any case: the second half costs 64 ragged sequences nothing (74.1 us), 24 compressed
// contexts 48.1 -> 48.5, the smallest call 9.7 -> 9.8.  fp32 caches use the fp32 matrix
// instructions.
#include "serve.h"

namespace gkv {

constexpr int PA_OCC = 3;          // waves a SIMD
// The last chunk of a row joins PA_JOIN states at a time (32 are up to a fifth slower, 16 the
// same; four dims a lane instead of two joins 16 heads faster, 128K tokens of one KV head 48 us
// instead of 55, and the others slower).
constexpr int PA_JOIN = 8;

static size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

// Workspace: a ticket word for every row and group of heads, then per chunk and head
// (max, sum), then the partial sums [chunk][hpg][d].
struct PagedWs {
  unsigned long long* ticket;
  unsigned long long* ml;
  float* o;
  size_t bytes;
};
static PagedWs paged_view(void* base, const PageDims& pg) {
  const size_t R = (size_t)pg.n_seq * pg.G, chunks = R + PA_TARGET;
  char* p = (char*)base;
  PagedWs w;
  size_t o = 0;
  w.ticket = (unsigned long long*)(p + o);
  o += al256(R * ((pg.hpg + PA_HEADS - 1) / PA_HEADS) * 8);
  w.ml = (unsigned long long*)(p + o);
  o += al256(chunks * pg.hpg * 8);
  w.o = (float*)(p + o);
  o += chunks * pg.hpg * pg.d * 4;
  w.bytes = o;
  return w;
}
size_t paged_ws_bytes(const PageDims& pg) { return paged_view(nullptr, pg).bytes; }
int64_t paged_items(const PageDims& pg) {
  return ((int64_t)pg.n_seq * pg.G + PA_TARGET) * ((pg.hpg + PA_HEADS - 1) / PA_HEADS);
}

// Tickets.  The chunks of a row count themselves in its word, PA_BASE, PA_BASE + 1, ...;
// the one that makes the count whole finds PA_BASE + parts - 1, and its counting sets the
// word to 0.  What a word holds before is no count: anything below PA_BASE is raised to it
// first, and counting on anything past the end gives 0, whoever did it counting again.
// So the workspace needs no clearing, and every call leaves the words it used at 0.  (The
// numbers from PA_BASE + 1 to PA_BASE + parts - 1, at most PA_BASE + PA_TARGET, would be taken
// for a count, and nothing here can tell them from one: the header excludes them.  Calls that
// overlap leave them, and nothing else does.)
// States are written and read with device-coherent operations, and a wait for the writes
// stands between them and the ticket, so no fence is needed, which on this chip would
// write back and invalidate the L2 of the XCD.  (Counting by compare-and-swap took the 40
// chunks of a row 20 us, one after the other.)
constexpr unsigned long long PA_BASE = 0x7fffffffffff0000ull;
static_assert(PA_TARGET <= 0xfff, "the words that the header excludes");
__device__ __forceinline__ bool last_of(unsigned long long* word, int parts) {
  const unsigned long long end = PA_BASE + parts - 1;
  unsigned long long was;
  do {
    __hip_atomic_fetch_max(word, PA_BASE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    was = __builtin_amdgcn_atomic_inc64((unsigned long*)word, end, __ATOMIC_RELAXED, "agent");
  } while (was > end || was < PA_BASE);       // below: put to 0 by another between the two steps
  return was == end;
}
// the thread's stores are where every other workgroup sees them
__device__ __forceinline__ void stores_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ unsigned long long pair_bits(float a, float b) {
  return (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32;
}
__device__ __forceinline__ float2 pair_of(unsigned long long x) {
  return make_float2(__uint_as_float((uint32_t)x), __uint_as_float((uint32_t)(x >> 32)));
}
__device__ __forceinline__ void put_agent(unsigned long long* p, unsigned long long x) {
  __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ int64_t held_count(const PrefixView& px, int64_t row, int64_t& start) {
  int64_t s = px.start[row], c = px.count[row];
  s = s < 0 ? 0 : (s > px.rows ? px.rows : s);
  c = c < 0 ? 0 : (c > px.rows - s ? px.rows - s : c);
  start = s;
  return c > PAGED_ROWS ? PAGED_ROWS : c;
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
// with the search, 403 without).
template <int TILE, bool PREFIX>
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
  int first = 0, size;
  if (units <= 64) {
    first = tiles(lane);
    size = chunk_tiles((uint64_t)(uint32_t)__builtin_amdgcn_readlane(scan_wave(first), 63) * mult, room);
  } else {
    __shared__ uint64_t part[PA_W];
    __shared__ int most[PA_W];
    uint64_t sum = 0;
    int mx = 0;
    for (int u = threadIdx.x; u < units; u += PA_T) {
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
    for (int i = 0; i < PA_W; ++i) { sum += part[i]; mx = max(mx, most[i]); }
    size = __builtin_amdgcn_readfirstlane(chunk_tiles(sum * mult, room));
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
      const int n = u0 ? tiles(u0 + lane) : first, x = n ? chunks_of(n, size, join) : 0;
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

template <typename T, int D, int NS, bool PREFIX>
__global__ __launch_bounds__(PA_T, PA_OCC) void k_paged(PageDims pg, int64_t q_tok, const T* __restrict__ q,
                                                   const T* __restrict__ Kp, const T* __restrict__ Vp,
                                                   const int32_t* __restrict__ table, const int32_t* __restrict__ len,
                                                   PrefixView px, T* __restrict__ out, float* __restrict__ lse, PagedWs ws) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int TILE = 16 * NS;
  constexpr int E = 16 / (int)sizeof(T);      // elements of 16 bytes
  constexpr int KC = D / 4 / E;               // 16-byte pieces of a lane's quarter of a key
  constexpr int VD = BF ? D / 16 : 4;         // neighbouring dims of a lane
  constexpr int VB = BF ? 1 : D / 64;         // ... in so many places of the row
  constexpr int VW = VD * (int)sizeof(T) / 4; // words of one place
  __shared__ float sM[PA_W][PA_HEADS], sL[PA_W][PA_HEADS];
  __shared__ __align__(16) float sO[PA_W][PA_HEADS][D + 4];      // rows start in other banks
  __shared__ int joins;
  // groups of 16 query heads of one chunk are neighbours: they read the same keys
  const int groups = (pg.hpg + PA_HEADS - 1) / PA_HEADS;
  const int bid = groups > 1 ? blockIdx.x / groups : blockIdx.x, group = groups > 1 ? blockIdx.x % groups : 0;
  Chunk ck;
  const int places = groups > 1 ? gridDim.x / groups : gridDim.x;
  if (!find_chunk<TILE, PREFIX>(pg, px, len, bid, places, join_cost(pg.hpg, D), ck)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g4 = lane >> 4;
  const int h0 = group * PA_HEADS, heads = min(PA_HEADS, pg.hpg - h0);
  const T* PK = (const T*)px.K;
  const T* PV = (const T*)px.V;
  constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;
  const float scale = 1.0f / sqrtf((float)D);
  const int seq = ck.b, kv = ck.g;
  const int64_t row = (int64_t)seq * pg.G + kv;
  const int64_t n_page = held_len(pg, len[seq]);
  int64_t p_start = 0, n_pack = 0;
  if constexpr (PREFIX) n_pack = held_count(px, row, p_start);
  const int pack_tiles = (int)((n_pack + TILE - 1) / TILE);

  // the group's queries: lane (head i16, quarter g4) holds pieces g4, g4 + 4, ... of the row
  uint4 qv[KC];
#pragma unroll
  for (int s = 0; s < KC; ++s)
    qv[s] = i16 < heads ? *(const uint4*)(q + seq * q_tok + ((int64_t)kv * pg.hpg + h0 + i16) * D + (4 * s + g4) * E)
                        : make_uint4(0, 0, 0, 0);

  // One tile's keys and values: the next tile's keys are asked for when the products with
  // the present ones are formed, the next values likewise, so the registers of one tile
  // keep a tile's loads in flight nearly all the time and leave room for a third wave.
  uint4 tk[NS][KC];
  uint32_t tv[NS][4][VB][VW];
  float lm[PREFIX ? NS : 1][4];   // log m of packed entries
  struct Where {                  // of a tile, the same for the wave: elements, entries there are
    int64_t at[NS], lm;
    int n[NS];
    bool packed;
  };
  const int32_t* tab = table + (int64_t)seq * pg.width;
  auto where = [&](int ti) __attribute__((always_inline)) {
    Where r;
    r.packed = PREFIX && ti < pack_tiles;
    r.lm = 0;
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      const int64_t e = (int64_t)(r.packed ? ti : ti - pack_tiles) * TILE + 16 * h;
      int64_t left = (r.packed ? n_pack : n_page) - e, at = 0;
      if (!r.packed && left > 0) {
        at = page_row(pg, tab[e >> pg.shift], kv, (int)(e & (((int64_t)1 << pg.shift) - 1)));
        if (at < 0) left = 0;
      } else if (r.packed) {
        at = (p_start + e) * D;
        if (h == 0) r.lm = p_start + e;
      }
      r.n[h] = left > 16 ? 16 : (left < 0 ? 0 : (int)left);
      r.at[h] = at;
    }
    return r;
  };
  // a page holds all 16 rows, written or not; the packed arrays may end behind the last
  // entry, which absent ones read in place of their own
  constexpr uint32_t RB = D * sizeof(T);
  auto load_keys = [&](const Where& t) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      if (t.n[h] == 0) {
#pragma unroll
        for (int s = 0; s < KC; ++s) tk[h][s] = make_uint4(0, 0, 0, 0);
        continue;
      }
      const char* base = (const char*)((t.packed ? PK : Kp) + t.at[h]);
      const uint32_t r = PREFIX && t.packed ? min(i16, t.n[h] - 1) : i16;
#pragma unroll
      for (int s = 0; s < KC; ++s) tk[h][s] = *(const uint4*)(base + (r * RB + 16 * g4) + 64 * s);
    }
  };
  auto load_values = [&](const Where& t) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      if (t.n[h] == 0) {
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int p = 0; p < VB; ++p)
#pragma unroll
            for (int x = 0; x < VW; ++x) tv[h][r][p][x] = 0;
      } else {
        const char* base = (const char*)((t.packed ? PV : Vp) + t.at[h]);
        auto rows = [&](auto row) __attribute__((always_inline)) {
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int p = 0; p < VB; ++p) {
              const char* x = base + (row(r) * RB + VD * sizeof(T) * i16) + 64 * sizeof(T) * p;
              if constexpr (VW == 4) {
                const uint4 u = *(const uint4*)x;
                tv[h][r][p][0] = u.x; tv[h][r][p][1] = u.y; tv[h][r][p][2] = u.z; tv[h][r][p][3] = u.w;
              } else {
                const uint2 u = *(const uint2*)x;
                tv[h][r][p][0] = u.x; tv[h][r][p][1] = u.y;
              }
            }
        };
        if (PREFIX && t.packed && t.n[h] < 16) rows([&](int r) { return (uint32_t)min(4 * g4 + r, t.n[h] - 1); });
        else rows([&](int r) { return (uint32_t)(4 * g4 + r); });
      }
      if constexpr (PREFIX) {
        if (t.packed) {
          const float* lp = px.logm + (t.lm + 16 * h) + 4 * g4;
          if (t.n[h] == 16) {
            __builtin_memcpy(lm[h], lp, 16);
          } else {
#pragma unroll
            for (int r = 0; r < 4; ++r) lm[h][r] = 4 * g4 + r < t.n[h] ? lp[r] : -INFINITY;
          }
        }
      }
    }
  };

  f32x4 o[VB][VD];
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int j = 0; j < VD; ++j) o[p][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;               // of head i16; l: this lane's entries only

  int ti = ck.t0 + w;
  Where now{}, next{};
  if (ti < ck.t1) {
    now = where(ti);
    load_keys(now);
    load_values(now);
  }
  for (; ti < ck.t1; ti += PA_W) {
    const bool more = ti + PA_W < ck.t1;
    if (more) next = where(ti + PA_W);
    float x[NS][4];
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f}, odd = acc;       // fp32: two chains, which round half as often
#pragma unroll
      for (int s = 0; s < KC; ++s) {
        if constexpr (BF) {
          acc = mfma_bf16_16x16x32(pk8(tk[h][s]), pk8(qv[s]), acc);
        } else {
          const uint32_t a[4] = {tk[h][s].x, tk[h][s].y, tk[h][s].z, tk[h][s].w};
          const uint32_t b[4] = {qv[s].x, qv[s].y, qv[s].z, qv[s].w};
#pragma unroll
          for (int i = 0; i < 4; i += 2) {
            acc = mfma_f32_16x16x4(__uint_as_float(a[i]), __uint_as_float(b[i]), acc);
            odd = mfma_f32_16x16x4(__uint_as_float(a[i + 1]), __uint_as_float(b[i + 1]), odd);
          }
        }
      }
      if constexpr (!BF) acc += odd;
#pragma unroll
      for (int r = 0; r < 4; ++r) x[h][r] = acc[r] * scale;
    }
    if (more) load_keys(next);
    bool all = !now.packed;
#pragma unroll
    for (int h = 0; h < NS; ++h) all &= now.n[h] == 16;
    if (!all) {                   // absent entries and those masked by their log m
      bool none[NS][4], any = false;
#pragma unroll
      for (int h = 0; h < NS; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          none[h][r] = 4 * g4 + r >= now.n[h];
          if (PREFIX && now.packed) {
            none[h][r] = lm[h][r] == -INFINITY;
            x[h][r] += lm[h][r];
          }
          any |= none[h][r];
        }
      if (__any(any)) {
#pragma unroll
        for (int h = 0; h < NS; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            x[h][r] = none[h][r] ? -INFINITY : x[h][r];
#pragma unroll
            for (int p = 0; p < VB; ++p)
#pragma unroll
              for (int i = 0; i < VW; ++i) tv[h][r][p][i] = none[h][r] ? 0 : tv[h][r][p][i];     // 0 times an infinity is not 0
          }
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
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx);
      const float c = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * LOG2E);
      m = mn;
      l *= c;
#pragma unroll
      for (int p = 0; p < VB; ++p)
#pragma unroll
        for (int j = 0; j < VD; ++j) o[p][j] *= c;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    float pr[NS][4];
#pragma unroll
    for (int h = 0; h < NS; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float y = (x[h][r] - ms) * LOG2E;
        pr[h][r] = __builtin_amdgcn_exp2f(y);
        // fp32: what the product lost, to first order
        if (!BF && pr[h][r] > 0.f) pr[h][r] = __builtin_fmaf(pr[h][r], __builtin_fmaf(x[h][r] - ms, LOG2E, -y) * LN2, pr[h][r]);
        l += pr[h][r];
      }
    if constexpr (BF) {
      // Each weight in two parts, its upper 16 bits and the rest rounded: off by at most 2^-15 of
      // itself.  The rest is at least 2^-16 of the weight, never 0 or negative where the weight is
      // not, so that an infinite value stays what it is.
      static_assert(NS == 2, "32 entries a product");
      uint32_t pb[NS][2], pl[NS][2];
#pragma unroll
      for (int h = 0; h < NS; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float a = pr[h][2 * i], b = pr[h][2 * i + 1];
          const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
          pb[h][i] = __builtin_amdgcn_perm(ub, ua, 0x07060302u);
          pl[h][i] = pack_bf16(fmaxf(a - __uint_as_float(ua & 0xffff0000u), a * 0x1p-16f),
                               fmaxf(b - __uint_as_float(ub & 0xffff0000u), b * 0x1p-16f));
        }
#pragma unroll
      for (int j = 0; j < VD; ++j) {
        const uint32_t sel = (j & 1) ? 0x07060302u : 0x05040100u;
        uint32_t a[NS][2];
#pragma unroll
        for (int h = 0; h < NS; ++h)
#pragma unroll
          for (int r = 0; r < 2; ++r)
            a[h][r] = __builtin_amdgcn_perm(tv[h][2 * r + 1][0][j / 2], tv[h][2 * r][0][j / 2], sel);
        const auto v8 = pk8(make_uint4(a[0][0], a[0][1], a[1][0], a[1][1]));
        o[0][j] = mfma_bf16_16x16x32(v8, pk8(make_uint4(pl[0][0], pl[0][1], pl[1][0], pl[1][1])), o[0][j]);
        o[0][j] = mfma_bf16_16x16x32(v8, pk8(make_uint4(pb[0][0], pb[0][1], pb[1][0], pb[1][1])), o[0][j]);
      }
    } else {
#pragma unroll
      for (int h = 0; h < NS; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int p = 0; p < VB; ++p)
#pragma unroll
            for (int j = 0; j < VD; ++j)
              o[p][j] = mfma_f32_16x16x4(__uint_as_float(tv[h][r][p][j]), pr[h][r], o[p][j]);
    }
    if (more) {
      load_values(next);
      now = next;
    }
  }
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int j = 0; j < VD; ++j) mfma_done(o[p][j]);
  l = col_sum4(l);
  // row 4 g4 + r of product (p, j) is dimension 64 p + VD (4 g4 + r) + j, column i16 the head
  if (g4 == 0) { sM[w][i16] = m; sL[w][i16] = l; }
  if (i16 < heads) {
#pragma unroll
    for (int p = 0; p < VB; ++p)
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int j = 0; j < VD; j += 4)
          *(float4*)&sO[w][i16][64 * p + VD * (4 * g4 + r) + j] = make_float4(o[p][j][r], o[p][j + 1][r], o[p][j + 2][r], o[p][j + 3][r]);
  }
  sync_after_lds_stores();
  auto finish = [&](int h, int dd, float M, float S, float O0, float O1) {
    const int64_t hd = (int64_t)seq * pg.H + (int64_t)kv * pg.hpg + h0 + h;
    stf(out, hd * D + dd, S > 0.f ? O0 / S : S);                  // nothing: 0; NaN stays
    stf(out, hd * D + dd + 1, S > 0.f ? O1 / S : S);
    if (lse && dd == 0) lse[hd] = M + logf(S);
  };
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
  const int64_t place = (int64_t)bid * pg.hpg + h0;
  for (int i = tid; i < heads * (D / 2); i += PA_T) {
    const int h = i / (D / 2), dd = 2 * (i % (D / 2));
    float M = -INFINITY, S = 0.f, O0 = 0.f, O1 = 0.f;
#pragma unroll
    for (int x = 0; x < PA_W; ++x) add(M, S, O0, O1, sM[x][h], sL[x][h], sO[x][h][dd], sO[x][h][dd + 1]);
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
  if (tid == 0) joins = last_of(ws.ticket + row * groups + group, ck.chunks);
  sync_after_lds_stores();
  if (!joins) return;
  // A head's pairs of dims lie on LH neighbouring lanes, which hold the (max, sum) of LH
  // chunks at a time, one each, and pass the weights round.
  constexpr int LH = D / 2;
  const int64_t base = (int64_t)(bid - ck.c) * pg.hpg + h0;              // the row's first chunk
  for (int i = tid; i < (heads * LH + 63) / 64 * 64; i += PA_T) {               // whole waves
    const int h = min(i / LH, heads - 1), sub = i % LH, dd = 2 * sub;
    float M = -INFINITY, S = 0.f, O0 = 0.f, O1 = 0.f;
    for (int b0 = 0; b0 < ck.chunks; b0 += LH) {
      const int nb = min(ck.chunks - b0, LH);
      const unsigned long long* src = (const unsigned long long*)(ws.o + (base + (int64_t)b0 * pg.hpg + h) * D + dd);
      const int64_t step = (int64_t)pg.hpg * LH;
      unsigned long long ov[PA_JOIN];
      auto load = [&](int c0) {                 // past the last: that one again
#pragma unroll
        for (int c = 0; c < PA_JOIN; ++c) ov[c] = ld_agent(src + min(c0 + c, nb - 1) * step);
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
      for (int c0 = 0; c0 < nb; c0 += PA_JOIN) {
        if (c0) load(c0);
#pragma unroll
        for (int c = 0; c < PA_JOIN; ++c) {
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

hipError_t launch_paged(const PageDims& pg, int64_t q_tok, const void* q, const void* Kp, const void* Vp,
                        const int32_t* table, const int32_t* len, const PrefixView& px, void* out, float* lse, void* ws,
                        hipStream_t st) {
  const PagedWs v = paged_view(ws, pg);
  const int64_t R = (int64_t)pg.n_seq * pg.G;                   // rows
  auto go = [&](auto type, auto dim, auto sub) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, NS = decltype(sub)::value;
    const int64_t room = chunk_room(pg, px.K ? px.rows : 0, 16 * NS);
    const dim3 grid((unsigned)((R + room) * ((pg.hpg + PA_HEADS - 1) / PA_HEADS)));
    if (px.K)
      hipLaunchKernelGGL((k_paged<T, D, NS, true>), grid, dim3(PA_T), 0, st, pg, q_tok, (const T*)q, (const T*)Kp, (const T*)Vp, table,
                         len, px, (T*)out, lse, v);
    else
      hipLaunchKernelGGL((k_paged<T, D, NS, false>), grid, dim3(PA_T), 0, st, pg, q_tok, (const T*)q, (const T*)Kp, (const T*)Vp, table,
                         len, px, (T*)out, lse, v);
    return hipGetLastError();
  };
  using std::integral_constant;
  if (pg.dtype == GRACEKV_BF16)
    return pg.d == 128 ? go(uint16_t{}, integral_constant<int, 128>{}, integral_constant<int, 2>{})
                       : go(uint16_t{}, integral_constant<int, 64>{}, integral_constant<int, 2>{});
  return pg.d == 128 ? go(float{}, integral_constant<int, 128>{}, integral_constant<int, 1>{})
                     : go(float{}, integral_constant<int, 64>{}, integral_constant<int, 2>{});
}

}  // namespace gkv
