// Attention of one token of every sequence over packed entries that groups of sequences share.
//
// Group s has the sequences [cu[s], cu[s+1]) and, of KV head g, the entries [start, start + count) of
// (s, g): every query head of g of every sequence of the group attends to all of them,
//   o = sum_j softmax_j(q.k_j / sqrt(d) + log m_j) v_j,  lse = log sum_j exp(...)
// (no entry: 0 and -inf).  Both are fp32: a state that another attention joins to its own.
//
// The rows that share keys, hpg of every sequence of the group, fill the tiles of a matrix product, so
// the entries are gone through once a row tile instead of once a sequence.  One pass with a running maximum and
// sum; every entry has a log m, and one of -inf has no weight: its value is replaced by 0, since 0 times an
// infinity is not 0.  A row tile's entries are cut into chunks, as many as fill the chip, found on
// the device by a scan over the groups' lengths (find_item).  Three kernels, chosen by shared_plan (groups.h):
//
// k_shared_few, 16 rows a workgroup, for little work: bound by latency.  Its waves have entries of their own, nothing is in LDS
// before they are merged, and the last of a row tile's chunks joins the states (tickets.h), so that there
// is one launch.  16 sequences over 2048 entries a head, 8 KV heads of 128, 32 query heads 14.1 us.
//
// k_shared_bf, 64 or 128 rows: bound by what feeds the matrix units.  Products are transposed, keys and values go
// straight into LDS, as in prompt.hip.  64 sequences over 16384 entries, heads as above (256 rows a KV head in two
// tiles, a chunk a CU) take 45 us: 30 in the loop, 4 to launch and find a chunk, 4 to write the states and 7 for
// k_shared_join.  Of a step of 128 keys a wave has 1770 cycles of logits (reads of LDS, each wave all of the keys), 720 of issuing the
// next tile's loads, 1250 of softmax and the weights' parts, 1350 of values, 170 of waiting at the barrier.  Tried and slower, with
// weights in one part: tiles of 64 keys in four stages, logits a tile ahead
// (43.7 us for 41.5), twice the chunks (54 for 41), four waves of 64 rows each, which read LDS half as often (50
// for 39: one wave a SIMD), joining in the same launch, by the chunks' workgroups in slices of the rows (40, and more where chunks are many).
//
// k_shared_f32, 64 rows: the fp32 matrix instructions, tiles of 32 keys through registers into LDS.
//
// The latter two leave states, megabytes of them, to k_shared_join, a second launch in which the whole chip
// reads them and not one workgroup a row tile.
//
// bf16 weights are held in two bf16 parts for the second product, by both kernels that have it: off by at most 2^-15 of themselves.
// Which kernel a call takes goes by the work and by rows of the arrays that are no concern of the caller's, and the result is fp32, so
// they are not held in fewer bits where products are the bound: one part, off by 2^-8, left 64 sequences over 16384 entries
// 9.5e-4 of the norm away from fp32 arithmetic, two 0.7e-4, for 45 us instead of 40.
#include <algorithm>

#include "tickets.h"
#include "tiles.h"

namespace gkv {

constexpr int SF_OCC = 3;                      // few rows: waves a SIMD
constexpr int SF_JOIN = 8;                     // ... and states that the last of a tile's chunks joins at a time
constexpr float SF_COST = PA_COST;             // ... and what joining one costs, as over pages, in steps of a tile, at d = 64 (chunks_of)
constexpr float SH_LAG = 8.f, SH_TOP = 256.f;  // as in prompt.hip: base-2 units, and as a factor
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

int64_t shared_items(const SharedDims& sd) { return most_tiles(sd, 16) * sd.G + 1024; }   // no plan has as many

// Workspace: where every row's states are, or a ticket word of every row tile, then per place and row (max, sum) and
// the weighted values.
struct SharedWs {
  int4* info;
  unsigned long long* ticket;
  int step;                    // words from ticket to ticket
  float2* ml;
  float* o;
  size_t bytes;
};
static SharedWs shared_view(void* base, const SharedDims& sd, const SharedPlan& p) {
  SharedWs w;
  size_t o = 0;
  w.info = (int4*)base;
  w.ticket = (unsigned long long*)base;               // few rows: in place of the other
  w.step = p.tiles <= 4096 ? 16 : 1;
  o += al256(p.few ? (size_t)p.tiles * 8 * w.step : (size_t)sd.n_seq * sd.H * 16);
  w.ml = (float2*)((char*)base + o);
  o += al256((size_t)p.places * p.rows * 8);
  w.o = (float*)((char*)base + o);
  o += (size_t)p.places * p.rows * sd.d * 4;
  w.bytes = o;
  return w;
}
// (of any kernel: how many entries there are is told with the call)
size_t shared_ws_bytes(const SharedDims& sd) {
  size_t n = 0;
  for (bool few : {false, true})
    for (int waves : {4, 8})
      if (few || waves == 4 || sd.dtype == GRACEKV_BF16) n = std::max(n, shared_view(nullptr, sd, plan_of(sd, few, waves)).bytes);
  return n;
}

// What a workgroup works on: key tiles [t0, t1), chunk c of `chunks`, of row tile `tile` of (group b, KV head g)
struct Item {
  int b, g, tile, tiles, c, chunks, t0, t1, id;
  int a, n;                    // the group's sequences
  int n_keys;
  int64_t p_start;             // ... and entries
};

// The item of workgroup blockIdx.x; false where there is none.  Units are (group, KV head);
// every wave looks at 64 of them at a time.
template <int ROWS, int KEYS, int LEAST, int W, typename F>
__device__ __forceinline__ bool find_item(const SharedDims& sd, const int32_t* cu, const PrefixView& px, int room, F chunks_for, Item& it) {
  const int lane = threadIdx.x & 63, units = sd.n_group * sd.G;
  // row tiles of unit u, and key tiles of each
  Span sp{0, 0};
  int64_t start = 0, count = 0;
  auto shape = [&](int u, int& mt, int& n) {
    mt = n = 0;
    if (u >= units) return;
    sp = span_of(cu, u / sd.G, sd.n_seq);
    mt = tiles_of_group(sd, sp.n, ROWS);
    count = held_count(px, u, start);
    n = (int)((count + KEYS - 1) / KEYS);
    if (n == 0) n = 1;                 // its zeros are written too
  };
  auto sum64 = [&](uint64_t v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
  };
  int mt, n;
  uint64_t total = 0;
  if (units <= 64) {
    shape(lane, mt, n);
    total = sum64((uint64_t)mt * n);
  } else {
    __shared__ uint64_t part[W];
    for (int u = threadIdx.x; u < units; u += 64 * W) {
      shape(u, mt, n);
      total += (uint64_t)mt * n;
    }
    total = sum64(total);
    if (lane == 0) part[threadIdx.x >> 6] = total;
    sync_after_lds_stores();
    total = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) total += part[i];
    shape(lane, mt, n);
  }
  const int size = __builtin_amdgcn_readfirstlane(shared_chunk(total, room, LEAST));
  int id = blockIdx.x, base = 0;
#pragma unroll 1
  for (int u0 = 0; u0 < units; u0 += 64) {
    if (u0) shape(u0 + lane, mt, n);
    const int ch = n ? chunks_for(n, size) : 0;
    const int64_t all64 = (int64_t)mt * ch;
    const int x = all64 > (1 << 24) ? 1 << 24 : (int)all64;
    int to = x;                          // inclusive sum over the lanes: at most 2^30
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(to, o, 64);
      if (lane >= o) to += y;
    }
    const int all = base + __builtin_amdgcn_readlane(to, 63);
    if (units <= 64) {
      id = item_of(id, all, gridDim.x);
      if (id < 0) return false;
    }
    if (id < all) {
      const int at = __popcll(__ballot(base + to <= id));       // the unit's lane
      const int u = u0 + at;
      it.tiles = __builtin_amdgcn_readlane(mt, at);
      it.chunks = __builtin_amdgcn_readlane(ch, at);
      const int tn = __builtin_amdgcn_readlane(n, at);
      const int local = id - base - (__builtin_amdgcn_readlane(to, at) - __builtin_amdgcn_readlane(x, at));
      it.b = u / sd.G;
      it.g = u % sd.G;
      it.c = local / it.tiles;
      it.tile = local % it.tiles;
      const int each = tn / it.chunks, more = tn % it.chunks;     // the first `more` take one more
      it.t0 = it.c * each + min(it.c, more);
      it.t1 = it.t0 + each + (it.c < more);
      it.id = id;
      it.a = __builtin_amdgcn_readlane((int)sp.a, at);
      it.n = __builtin_amdgcn_readlane((int)sp.n, at);
      it.n_keys = __builtin_amdgcn_readlane((int)count, at);
      it.p_start = (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)start, at) |
                             (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(start >> 32), at) << 32);
      return true;
    }
    base = all;
  }
  return false;
}

// chunks of a row tile with n key tiles, `size` or fewer of them each
struct {
  __device__ int operator()(int n, int size) const { return n / size + (n % size != 0); }
} constexpr whole_chunks{};

// the rows of an item's tile: the lane's row, and where its query and its result lie
struct Row {
  int row, rows;               // of the group
  int64_t hd;                  // sequence * H + head
};
__device__ __forceinline__ Row row_of(const SharedDims& sd, const Item& it, int R, int r, int64_t& seq) {
  Row x;
  x.rows = it.n * sd.hpg;
  x.row = it.tile * R + r;
  const int c = min(x.row, x.rows - 1), tok = (int)((uint32_t)c / (uint32_t)sd.hpg);
  seq = it.a + tok;
  x.hd = seq * sd.H + (int64_t)it.g * sd.hpg + (c - tok * sd.hpg);
  return x;
}
// the row tile's place among all of them
__device__ __forceinline__ int64_t slot_of(const SharedDims& sd, const Item& it, int R) {
  return (int64_t)(first_tile(sd, it.a, it.b, R) + it.tile) * sd.G + it.g;
}

// Many rows a group: W waves, pairs of them to the same 32 rows with 32 NU keys each of a tile.  One tile is in
// LDS and the next on its way.
template <int D, int W>
__global__ __launch_bounds__(64 * W, W / 4) void k_shared_bf(SharedDims sd, int room, const uint16_t* __restrict__ q,
                                                             const int32_t* __restrict__ cu, PrefixView px, float* __restrict__ out,
                                                             float* __restrict__ lse, SharedWs ws) {
  constexpr int SPLIT = 2, NU = 2, ROWS = 32 * W / SPLIT, KEYS = 32 * NU * SPLIT;
  constexpr int CH = D / 8;                     // 16-byte pieces of a row
  constexpr int RI = 64 / CH;                   // rows that one load of a wave brings
  constexpr int NI = KEYS / RI / W;             // such loads of a wave and array
  constexpr int KS = D / 16;                    // product steps over the dims
  constexpr int DT = D / 32;                    // 32-dim tiles of the output
  constexpr int V0 = KEYS * CH, L0 = 2 * V0;    // of a stage: keys, values, each wave's own copy of log m
  constexpr int STAGE = L0 + W * KEYS / 4;
  __shared__ __align__(16) uint4 st0[STAGE], st1[STAGE];      // of their own, so that loads into one and reads of the other are told apart
  Item it;
  if (!find_item<ROWS, KEYS, 1, W>(sd, cu, px, room, whole_chunks, it)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i32 = lane & 31, half = lane >> 5;
  const int rw = w / SPLIT, kw = w % SPLIT;     // the wave's 32 rows, its 32 keys of a tile
  int64_t seq;
  const Row me = row_of(sd, it, ROWS, 32 * rw + i32, seq);
  const int n_keys = it.n_keys;

  uint4 qv[KS];
  {
    const uint16_t* qp = q + seq * sd.q_tok + (me.hd - seq * sd.H) * D;
#pragma unroll
    for (int s = 0; s < KS; ++s) qv[s] = *(const uint4*)(qp + 16 * s + 8 * half);
  }
  // where the row's states will be, for the kernel that joins them
  if (it.c == 0 && kw == 0 && half == 0 && me.row < me.rows)
    ws.info[me.hd] = make_int4(it.id, it.chunks, it.tiles, 32 * rw + i32);
  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  float m = -INFINITY, l = 0.f;                 // what is subtracted, natural units; l: this lane's keys only
  const float root = sqrtf((float)D), scale = 1.f / root, sc2 = LOG2E / root;

  const uint16_t* kp = (const uint16_t*)px.K + it.p_start * D;
  const uint16_t* vp = (const uint16_t*)px.V + it.p_start * D;
  const float* lp = px.logm + it.p_start;
  const int t1 = n_keys > 0 ? it.t1 : it.t0;     // an empty row: its zeros only
  // Load i of a wave brings rows RI (w + W i) .. + RI - 1 straight into LDS (prompt.hip)
  const int lr = RI * w + lane / CH, lc = swz<D>(lr, lane % CH) - lr * CH;
  const int off = lr * D * 2 + lc * 16;
  constexpr int STEP = RI * W * D * 2;
  auto load_tile = [&](int t, uint4* to) __attribute__((always_inline)) {
    const int n = min(n_keys - t * KEYS, KEYS);
    const int64_t at = (int64_t)t * KEYS;
    const Buffer k = __builtin_amdgcn_make_buffer_rsrc((void*)(kp + at * D), 0, n * D * 2, 0x00020000);
    const Buffer v = __builtin_amdgcn_make_buffer_rsrc((void*)(vp + at * D), 0, n * D * 2, 0x00020000);
    const Buffer g = __builtin_amdgcn_make_buffer_rsrc((void*)(lp + at), 0, n * 4, 0x00020000);
#pragma unroll
    for (int i = 0; i < NI; ++i) buffer_load_lds(k, to + 64 * (w + W * i), off + i * STEP);
#pragma unroll
    for (int i = 0; i < NI; ++i) buffer_load_lds(v, to + V0 + 64 * (w + W * i), off + i * STEP);
#pragma unroll
    for (int i = 0; i < KEYS / 64; ++i)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(g, (__attribute__((address_space(3))) void*)(to + L0 + w * KEYS / 4 + 16 * i), 4, 4 * lane + 256 * i, 0, 0, 0);
  };
  constexpr int RB = 2 * D;
  int k_at = 16 * swz<D>(i32, half);
  const int v_at = 16 * swz<D>(4 * half + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
  // Below LOW, which only a mask is (-inf, the type's lowest value), log m is all of a logit: nothing beside
  // others, and where a row has seen no others, its weight is 1 at the largest and 0 else.  Units of the sums would
  // take it out of range.
  constexpr float LOW = -1e36f;
  auto log_m = [&](const uint4* tile, int u, float* lm) __attribute__((always_inline)) {
#pragma unroll
    for (int b = 0; b < 4; ++b) {                // register r: key 8 (r / 4) + 4 half + r % 4 of the wave's u-th 32
      const uint4 g = lds_at(tile, 16 * (L0 + w * KEYS / 4) + 4 * (32 * (NU * kw + u) + 4 * half + 8 * b));
      lm[4 * b] = __uint_as_float(g.x); lm[4 * b + 1] = __uint_as_float(g.y);
      lm[4 * b + 2] = __uint_as_float(g.z); lm[4 * b + 3] = __uint_as_float(g.w);
    }
  };
  auto step = [&](int t, uint4* cur, uint4* next) __attribute__((always_inline)) {
    // the wave's own loads of tile t are there, then everyone's; and everyone is done with tile t - 1
    loaded_barrier<0>();
    if (W == 4 && t + 1 < t1) load_tile(t + 1, next);
    uint4* cV = cur + V0;
    const int left = n_keys - t * KEYS;          // entries from this tile on
    const float* cL = (const float*)(cur + L0 + w * KEYS / 4);
    float lk[NU];                                // of the lane's keys
#pragma unroll
    for (int u = 0; u < NU; ++u) lk[u] = cL[32 * (NU * kw + u) + i32];
    bool low = false;                            // some log m is below LOW, or no number
#pragma unroll
    for (int i = 0; i < KEYS; i += 64) low |= i + lane < left && !(cL[i + lane] >= LOW);
    low = __any(low);                            // the same for every wave
    // log m comes into the sums by a product of its own, in their units and in three bf16 parts, which
    // hold it, with ones: read from LDS into every lane's sums it would take half as long again as the keys
    f32x16 s[NU];
    const uint32_t lower = half == 0 ? 0xffffffffu : 0u;
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      float g = fmaxf(lk[u], LOW) * root;
      const uint32_t hi = __float_as_uint(g) & 0xffff0000u;
      g -= __uint_as_float(hi);
      const uint32_t mid = __float_as_uint(g) & 0xffff0000u;
      g -= __uint_as_float(mid);
      const uint4 part = make_uint4((hi >> 16 | mid) & lower, (__float_as_uint(g) >> 16) & lower, 0, 0);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[u][r] = 0.f;
      s[u] = mfma_bf16_32x32x16(part, make_uint4(0x3f803f80u, 0x3f80u, 0, 0), s[u]);
      asm volatile("" : "+v"(k_at));             // eight places: formed anew, not held in registers
#pragma unroll
      for (int x = 0; x < KS; ++x) s[u] = mfma_bf16_32x32x16(lds_at(cur, (k_at ^ (32 * x)) + 32 * (NU * kw + u) * RB), qv[x], s[u]);
    }
    reads_ahead<NU * (KS + 1), 1, 8>();
#pragma unroll
    for (int u = 0; u < NU; ++u) mfma_done16(s[u]);
    // eight waves, which the products bound: behind the logits, whose reads the loads would meet (with weights in
    // one part 512 rows over 16384 entries 57.6 us in front of them, 55.0 behind); four wait for memory (4 rows over 65536 64 and 70)
    if (W == 8 && t + 1 < t1) load_tile(t + 1, next);
    if (left < KEYS) {
      asm volatile("");                          // (a branch: 64 selects in every tile otherwise)
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        const int rel = left - 32 * (NU * kw + u) - 4 * half;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[u][r] = 8 * (r / 4) + r % 4 >= rel ? -INFINITY : s[u][r];
      }
    }
    float most = -INFINITY;
    if (low) {
      for (int i = tid; i < KEYS * CH; i += 64 * W)        // no weight: a value of 0, whatever it was
        if (cL[i / CH] == -INFINITY) cV[i] = make_uint4(0, 0, 0, 0);       // a row's pieces stay in its places
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float lm[16];
        log_m(cur, u, lm);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (8 * (r / 4) + r % 4 < left - 32 * (NU * kw + u) - 4 * half && !(lm[r] >= LOW)) {
            most = fmaxf(most, lm[r]);
            s[u][r] = lm[r] < LOW ? -INFINITY : lm[r];
          }
      }
      sync_after_lds_stores();
    }
    float mx = s[0][0];
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[u][r]);
    mx = fmaxf(mx * scale, most);
    {
      const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if (__any(mx > m)) {                         // (prompt.hip on what is subtracted)
      const float mn = fmaxf(m, mx + SH_LAG * LN2);
      const float c = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((m - mn) * LOG2E);
      m = mn;
      l *= c;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= c;
    }
    float ms2 = m == -INFINITY ? 0.f : m * LOG2E;
    if (__any(m < LOW && m > -INFINITY)) {       // rows that have seen such entries only (so `low` is true, or the row's keys are none)
      if (m < LOW && m > -INFINITY) ms2 = 0.f;
#pragma unroll
      for (int u = 0; u < NU; ++u) {
        float lm[16];
        log_m(cur, u, lm);
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (m < LOW && m > -INFINITY)
            s[u][r] = 8 * (r / 4) + r % 4 < left - 32 * (NU * kw + u) - 4 * half && lm[r] == m ? 0.f : -INFINITY;
      }
    }
    uint4 pr[NU][2], pl[NU][2];                  // weights in two parts
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float e[8], f[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][8 * h + r], sc2, -ms2));
        l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
        // the second is what the first leaves and 2^-20 of the weight, so that an infinite value does not meet a 0 (a weight
        // below 2^-113 of one may give NaN for it)
#pragma unroll
        for (int r = 0; r < 8; ++r) f[r] = __builtin_fmaf(e[r], 1.f + 0x1p-20f, -upper(e[r]));
        pr[u][h] = make_uint4(uppers(e[0], e[1]), uppers(e[2], e[3]), uppers(e[4], e[5]), uppers(e[6], e[7]));
        pl[u][h] = make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
      }
    // product step x: keys 16 x + 8 (j / 4) + 4 half + j % 4 in place 8 half + j
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const int row = 32 * (NU * kw + u) + 16 * x;
          const uint2 a = lds_read_tr(cV, (v_at ^ (64 * d)) + row * RB);
          const uint2 b = lds_read_tr(cV, (v_at ^ (64 * d + 32)) + (row + 8) * RB);
          const uint4 v8 = make_uint4(a.x, a.y, b.x, b.y);
          o[d] = mfma_bf16_32x32x16(v8, pl[u][x], o[d]);
          o[d] = mfma_bf16_32x32x16(v8, pr[u][x], o[d]);
        }
    reads_ahead<2 * DT * NU, 2, 3, 2>();
  };
  if (it.t0 < t1) load_tile(it.t0, st0);
  for (int t = it.t0; t < t1; t += 2) {
    step(t, st0, st1);
    if (t + 1 < t1) step(t + 1, st1, st0);
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) mfma_done16(o[d]);
  {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  const bool mine = me.row < me.rows;
  // the two waves of the same rows join their states, each half of the dims, through the tiles' LDS
  static_assert(2 * STAGE * 16 >= W * 64 * 4 * 16 * DT, "a stage for half of the waves");
  __shared__ float2 sml[W][32];
  sync_after_lds_stores();
  auto sums = [&](int x) { return (float*)(x < W / 2 ? st0 : st1) + (x % (W / 2)) * 64 * 16 * DT; };
  float* so = sums(w);
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) so[64 * (16 * d + r) + lane] = o[d][r];
  if (half == 0) sml[w][i32] = make_float2(m, l);
  sync_after_lds_stores();
  if (!mine) return;
  const float2 x0 = sml[SPLIT * rw][i32], x1 = sml[SPLIT * rw + 1][i32];
  const float mm = fmaxf(x0.x, x1.x);
  const float f0 = x0.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x0.x - mm) * LOG2E), f1 = x1.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((x1.x - mm) * LOG2E);
  const float ll = (f0 == 0.f && x0.y == x0.y ? 0.f : x0.y * f0) + (f1 == 0.f && x1.y == x1.y ? 0.f : x1.y * f1);       // NaN stays
  // the result, or the place's state
  const int64_t place = (int64_t)it.id * ROWS + 32 * rw + i32;
  float* to = it.chunks > 1 ? ws.o + place * D : out + me.hd * D;
  const float inv = it.chunks > 1 ? 1.f : (ll > 0.f ? 1.f / ll : ll);    // no entry: the sums are 0; NaN stays
  const float *s0 = sums(SPLIT * rw), *s1 = sums(SPLIT * rw + 1);
#pragma unroll
  for (int d0 = 0; d0 < DT / 2; ++d0) {
    const int d = d0 + kw * (DT / 2);
    float a[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float y0 = s0[64 * (16 * d + r) + lane], y1 = s1[64 * (16 * d + r) + lane];
      a[r] = ((f0 == 0.f ? 0.f : y0 * f0) + (f1 == 0.f ? 0.f : y1 * f1)) * inv;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) *(float4*)(to + 32 * d + 8 * r + 4 * half) = make_float4(a[4 * r], a[4 * r + 1], a[4 * r + 2], a[4 * r + 3]);
  }
  if (kw == 0 && half == 0) {
    if (it.chunks > 1) ws.ml[place] = make_float2(mm, ll);
    // (with the sum in units of its largest weight, whose logarithm is small)
    else lse[me.hd] = mm == -INFINITY ? logf(ll) : (mm - SH_LAG * LN2) + logf(ll * SH_TOP);
  }
}

// 16 bytes of a state, written and read past the caches that only one XCD sees (the cache policy of a
// relaxed access of device scope)
constexpr int AGENT = 16;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ Buffer state_buffer(float* base, int n) {
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, 4 * n, 0x00020000);
}
__device__ __forceinline__ void put_agent16(Buffer b, int byte, const float* x) {
  const u32x4 v = {__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  __builtin_amdgcn_raw_buffer_store_b128(v, b, byte, 0, AGENT);
}
__device__ __forceinline__ float4 ld_agent16(Buffer b, int byte) {
  return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(b, byte, 0, AGENT));
}

// Few rows a group: 16 of them a workgroup, whose waves have a tile of 16 NS entries each at a time, keys
// straight from memory as the product's operand and values paired up in registers, as over pages
// (paged.hip), and no LDS before the waves are merged.  The last of a row tile's chunks joins them.
// Eight waves halve the states of longer rows, which is what four wait for (groups.h has both measured).
template <typename T, int D, int NS, int W>
__global__ __launch_bounds__(64 * W, W == 8 ? 2 : SF_OCC) void k_shared_few(SharedDims sd, int room, const T* __restrict__ q, const int32_t* __restrict__ cu,
                                                             PrefixView px, float* __restrict__ out, float* __restrict__ lse, SharedWs ws) {
  constexpr bool BF = sizeof(T) == 2;
  constexpr int ROWS = 16, TILE = 16 * NS;
  constexpr int E = 16 / (int)sizeof(T);      // elements of 16 bytes
  constexpr int KC = D / 4 / E;               // 16-byte pieces of a lane's quarter of a key
  constexpr int VD = BF ? D / 16 : 4;         // neighbouring dims of a lane
  constexpr int VB = BF ? 1 : D / 64;         // ... in so many places of the row
  constexpr int VW = VD * (int)sizeof(T) / 4; // words of one place
  __shared__ float sM[W][ROWS], sL[W][ROWS];
  __shared__ __align__(16) float sO[W][ROWS][D + 4];      // rows start in other banks
  __shared__ int joins;
  Item it;
  // (chunks of eight waves are counted in pairs of tiles)
  constexpr int PAIR = W / SH_W;
  const float join = SF_COST * (D / 64) / PAIR;
  if (!find_item<ROWS, TILE * PAIR, PA_MIN, W>(sd, cu, px, room, [&](int n, int size) { return chunks_of(n, size, join); }, it)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g4 = lane >> 4;
  const float scale = 1.0f / sqrtf((float)D);
  int64_t seq;
  const Row me = row_of(sd, it, ROWS, i16, seq);
  const int n_keys = it.n_keys;
  const T* kp = (const T*)px.K + it.p_start * D;
  const T* vp = (const T*)px.V + it.p_start * D;
  const float* lp = px.logm + it.p_start;
  uint4 qv[KC];                               // pieces g4, g4 + 4, ... of the row
#pragma unroll
  for (int s = 0; s < KC; ++s) qv[s] = *(const uint4*)(q + seq * sd.q_tok + (me.hd - seq * sd.H) * D + (4 * s + g4) * E);

  uint4 tk[NS][KC];
  uint32_t tv[NS][4][VB][VW];
  float lm[NS][4];
  constexpr uint32_t RB = D * sizeof(T);
  // entries behind the last one read that in place of their own
  auto load_keys = [&](int ti) __attribute__((always_inline)) {
    const char* base = (const char*)(kp + (int64_t)ti * TILE * D);
    const int last = n_keys - ti * TILE - 1;
#pragma unroll
    for (int h = 0; h < NS; ++h) {
      const uint32_t r = min(16 * h + i16, last);
#pragma unroll
      for (int s = 0; s < KC; ++s) tk[h][s] = *(const uint4*)(base + (r * RB + 16 * g4) + 64 * s);
    }
  };
  auto load_values = [&](int ti) __attribute__((always_inline)) {
    const char* base = (const char*)(vp + (int64_t)ti * TILE * D);
    const float* lb = lp + (int64_t)ti * TILE;
    const int last = n_keys - ti * TILE - 1;
#pragma unroll
    for (int h = 0; h < NS; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int e = 16 * h + 4 * g4 + r;
        const uint32_t at = min(e, last);
        lm[h][r] = lb[at];
        if (e > last) lm[h][r] = -INFINITY;
#pragma unroll
        for (int p = 0; p < VB; ++p) {
          const char* x = base + (at * RB + VD * sizeof(T) * i16) + 64 * sizeof(T) * p;
          if constexpr (VW == 4) {
            const uint4 u = *(const uint4*)x;
            tv[h][r][p][0] = u.x; tv[h][r][p][1] = u.y; tv[h][r][p][2] = u.z; tv[h][r][p][3] = u.w;
          } else {
            const uint2 u = *(const uint2*)x;
            tv[h][r][p][0] = u.x; tv[h][r][p][1] = u.y;
          }
        }
      }
  };
  f32x4 o[VB][VD];
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int j = 0; j < VD; ++j) o[p][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;               // of row i16, natural units; l: this lane's entries only
  const int t1 = n_keys > 0 ? min(it.t1 * PAIR, (n_keys + TILE - 1) / TILE) : 0;
  int ti = it.t0 * PAIR + w;
  if (ti < t1) {
    load_keys(ti);
    load_values(ti);
  }
  for (; ti < t1; ti += W) {
    const bool more = ti + W < t1;
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
    if (more) load_keys(ti + W);
    bool any = false;
#pragma unroll
    for (int h = 0; h < NS; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        any |= lm[h][r] == -INFINITY;
        x[h][r] += lm[h][r];
      }
    if (__any(any)) {             // absent entries and those without weight
#pragma unroll
      for (int h = 0; h < NS; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const bool none = lm[h][r] == -INFINITY;
          x[h][r] = none ? -INFINITY : x[h][r];
#pragma unroll
          for (int p = 0; p < VB; ++p)
#pragma unroll
            for (int i = 0; i < VW; ++i) tv[h][r][p][i] = none ? 0 : tv[h][r][p][i];     // 0 times an infinity is not 0
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
      // the second part is never 0 where the weight is not, so that an infinite value stays one (paged.hip)
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
          for (int r = 0; r < 2; ++r) a[h][r] = __builtin_amdgcn_perm(tv[h][2 * r + 1][0][j / 2], tv[h][2 * r][0][j / 2], sel);
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
            for (int j = 0; j < VD; ++j) o[p][j] = mfma_f32_16x16x4(__uint_as_float(tv[h][r][p][j]), pr[h][r], o[p][j]);
    }
    if (more) load_values(ti + W);
  }
  // the tile's ticket word is made ready now, for its chunks to count themselves in one step
  unsigned long long* ticket = ws.ticket + slot_of(sd, it, ROWS) * ws.step;
  if (it.chunks > 1 && tid == 0) raise(ticket);
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int j = 0; j < VD; ++j) mfma_done(o[p][j]);
  l = col_sum4(l);
  // row 4 g4 + r of product (p, j) is dimension 64 p + VD (4 g4 + r) + j, column i16 the row
  if (g4 == 0) { sM[w][i16] = m; sL[w][i16] = l; }
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int j = 0; j < VD; j += 4)
        *(float4*)&sO[w][i16][64 * p + VD * (4 * g4 + r) + j] = make_float4(o[p][j][r], o[p][j + 1][r], o[p][j + 2][r], o[p][j + 3][r]);
  sync_after_lds_stores();
  // from here a thread has eight dims of one row
  constexpr int LH = D / 8;
  const int r = tid / LH, c = 8 * (tid % LH);
  const Row at = row_of(sd, it, ROWS, r < ROWS ? r : 0, seq);
  const bool mine = r < ROWS && at.row < at.rows;
  float M = -INFINITY, S = 0.f, O[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) O[i] = 0.f;
  // state (m2, s2, a) onto (M, S, O): one of no entry has the maximum -inf and adds nothing, unless its
  // sum is no number
  auto add = [&](float m2, float s2, const float* a) {
    const float mn = fmaxf(M, m2);
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((M - mn) * LOG2E);
    const float g = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m2 - mn) * LOG2E);
    S = (f == 0.f && S == S ? 0.f : S * f) + (g == 0.f && s2 == s2 ? 0.f : s2 * g);
#pragma unroll
    for (int i = 0; i < 8; ++i) O[i] = (f == 0.f ? 0.f : O[i] * f) + (g == 0.f ? 0.f : a[i] * g);
    M = mn;
  };
  auto finish = [&] {
    const float inv = S > 0.f ? 1.f / S : S;                    // no entry: the sums are 0; NaN stays
    *(float4*)(out + at.hd * D + c) = make_float4(O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv);
    *(float4*)(out + at.hd * D + c + 4) = make_float4(O[4] * inv, O[5] * inv, O[6] * inv, O[7] * inv);
    if (c == 0) lse[at.hd] = M + logf(S);
  };
  if (mine) {
#pragma unroll
    for (int x = 0; x < W; ++x) {
      float a[8];
#pragma unroll
      for (int i = 0; i < 8; i += 4) *(float4*)(a + i) = *(const float4*)&sO[x][r][c + i];
      add(sM[x][r], sL[x][r], a);
    }
    if (it.chunks == 1) {
      finish();
    } else {
      const Buffer to = state_buffer(ws.o + (int64_t)it.id * ROWS * D, ROWS * D);
#pragma unroll
      for (int i = 0; i < 8; i += 4) put_agent16(to, 4 * (r * D + c + i), O + i);
      if (c == 0) put_agent((unsigned long long*)(ws.ml + (int64_t)it.id * ROWS + r), pair_bits(M, S));
    }
  }
  if (it.chunks == 1) return;
  stores_done();
  __syncthreads();
  if (tid == 0) joins = last_of<true>(ticket, it.chunks);
  sync_after_lds_stores();
  if (!joins || !mine) return;
  const int64_t first = it.id - it.c * it.tiles;          // the tile's chunks: places first + x * it.tiles
  M = -INFINITY; S = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) O[i] = 0.f;
  for (int c0 = 0; c0 < it.chunks; c0 += SF_JOIN) {
    unsigned long long ml[SF_JOIN];
    float4 ov[SF_JOIN][2];
#pragma unroll
    for (int x = 0; x < SF_JOIN; ++x) {            // past the last: that one again
      const int64_t id = first + (int64_t)min(c0 + x, it.chunks - 1) * it.tiles;
      const int64_t p = (id < gridDim.x ? id : gridDim.x - 1) * ROWS;        // (past the places only where groups descend: item_of)
      ml[x] = ld_agent((const unsigned long long*)(ws.ml + p + r));
      const Buffer from = state_buffer(ws.o + p * D, ROWS * D);
#pragma unroll
      for (int i = 0; i < 2; ++i) ov[x][i] = ld_agent16(from, 4 * (r * D + c + 4 * i));
    }
#pragma unroll
    for (int x = 0; x < SF_JOIN; ++x)
      if (c0 + x < it.chunks) {
        const float a[8] = {ov[x][0].x, ov[x][0].y, ov[x][0].z, ov[x][0].w, ov[x][1].x, ov[x][1].y, ov[x][1].z, ov[x][1].w};
        const float2 y = pair_of(ml[x]);
        add(y.x, y.y, a);
      }
  }
  finish();
}

// fp32: 16 rows a wave, fp32 matrix instructions
template <int D>
__global__ __launch_bounds__(SH_T, 2) void k_shared_f32(SharedDims sd, int room, const float* __restrict__ q, const int32_t* __restrict__ cu,
                                                        PrefixView px, float* __restrict__ out, float* __restrict__ lse, SharedWs ws) {
  constexpr int ROWS = 16 * SH_W, KEYS = 32;
  constexpr int CH = D / 4, NL = KEYS * CH / SH_T, LD = D + 4;
  constexpr int KC = D / 16, VB = D / 64;
  __shared__ __align__(16) float sK[KEYS * LD], sV[KEYS * LD], sL[KEYS];
  Item it;
  if (!find_item<ROWS, KEYS, 1, SH_W>(sd, cu, px, room, whole_chunks, it)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g4 = lane >> 4;
  int64_t seq;
  const Row me = row_of(sd, it, ROWS, 16 * w + i16, seq);
  const int n_keys = it.n_keys;
  if (it.c == 0 && g4 == 0 && me.row < me.rows) ws.info[me.hd] = make_int4(it.id, it.chunks, it.tiles, 16 * w + i16);

  float4 qv[KC];                                // pieces g4, g4 + 4, ... of the row
  {
    const float* qp = q + seq * sd.q_tok + (me.hd - seq * sd.H) * D;
#pragma unroll
    for (int s = 0; s < KC; ++s) qv[s] = *(const float4*)(qp + 16 * s + 4 * g4);
  }
  f32x4 o[VB][4];
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[p][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;                 // natural units; l: this lane's keys only
  const float scale = 1.f / sqrtf((float)D);
  const float* kp = (const float*)px.K + it.p_start * D;
  const float* vp = (const float*)px.V + it.p_start * D;
  const float* lp = px.logm + it.p_start;
  uint4 rk[NL], rv[NL];
  float rl = 0.f;
  // entries that are absent or have no weight: log m = -inf, and a value of 0
  auto load = [&](int t) {
    const int left = n_keys - t * KEYS;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int e = tid + SH_T * i, c = e % CH, j = e / CH;
      const int64_t at = ((int64_t)t * KEYS + j) * D + 4 * c;
      rk[i] = j < left ? *(const uint4*)(kp + at) : make_uint4(0, 0, 0, 0);
      rv[i] = j < left ? *(const uint4*)(vp + at) : make_uint4(0, 0, 0, 0);
    }
    if (tid < KEYS) rl = tid < left ? lp[(int64_t)t * KEYS + tid] : -INFINITY;
  };
  const int t1 = n_keys > 0 ? it.t1 : it.t0;
  if (it.t0 < t1) load(it.t0);
  for (int t = it.t0; t < t1; ++t) {
    sync_after_lds_stores();
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int e = tid + SH_T * i;
      *(uint4*)(sK + e / CH * LD + 4 * (e % CH)) = rk[i];
      *(uint4*)(sV + e / CH * LD + 4 * (e % CH)) = rv[i];
    }
    if (tid < KEYS) sL[tid] = rl;
    if (t + 1 < t1) load(t + 1);
    sync_after_lds_stores();
    bool none = false;
    if (lane < KEYS) none = sL[lane] == -INFINITY;
    if (__any(none)) {                          // the same for every wave
      for (int i = tid; i < KEYS * CH; i += SH_T)
        if (sL[i / CH] == -INFINITY) *(uint4*)(sV + i / CH * LD + 4 * (i % CH)) = make_uint4(0, 0, 0, 0);
      sync_after_lds_stores();
    }
    float x[KEYS / 16][4];
#pragma unroll
    for (int b = 0; b < KEYS / 16; ++b) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f}, odd = acc;       // two chains, which round half as often
#pragma unroll
      for (int s = 0; s < KC; ++s) {
        const float4 a = *(const float4*)(sK + (16 * b + i16) * LD + 16 * s + 4 * g4);
        acc = mfma_f32_16x16x4(a.x, qv[s].x, acc);
        odd = mfma_f32_16x16x4(a.y, qv[s].y, odd);
        acc = mfma_f32_16x16x4(a.z, qv[s].z, acc);
        odd = mfma_f32_16x16x4(a.w, qv[s].w, odd);
      }
      mfma_done(acc);
      mfma_done(odd);
      acc += odd;
      const float4 g = *(const float4*)(sL + 16 * b + 4 * g4);
      const float lg[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
      for (int r = 0; r < 4; ++r) x[b][r] = lg[r] == -INFINITY ? -INFINITY : acc[r] * scale + lg[r];
    }
    float mx = x[0][0];
#pragma unroll
    for (int b = 0; b < KEYS / 16; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[b][r]);
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
        for (int j = 0; j < 4; ++j) o[p][j] *= c;
    }
    const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int b = 0; b < KEYS / 16; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float y = (x[b][r] - ms) * LOG2E;
        float e = __builtin_amdgcn_exp2f(y);
        // what the product lost, to first order
        if (e > 0.f) e = __builtin_fmaf(e, __builtin_fmaf(x[b][r] - ms, LOG2E, -y) * LN2, e);
        l += e;
#pragma unroll
        for (int p = 0; p < VB; ++p) {
          const float4 a = *(const float4*)(sV + (16 * b + 4 * g4 + r) * LD + 64 * p + 4 * i16);
          o[p][0] = mfma_f32_16x16x4(a.x, e, o[p][0]);
          o[p][1] = mfma_f32_16x16x4(a.y, e, o[p][1]);
          o[p][2] = mfma_f32_16x16x4(a.z, e, o[p][2]);
          o[p][3] = mfma_f32_16x16x4(a.w, e, o[p][3]);
        }
      }
#pragma unroll
    for (int p = 0; p < VB; ++p) mfma_done(o[p]);
  }
  l = col_sum4(l);
  const bool mine = me.row < me.rows;
  const int64_t place = (int64_t)it.id * ROWS + 16 * w + i16;
  float* to = it.chunks > 1 ? ws.o + place * D : out + me.hd * D;
  auto sums = [&](float mm, float ll) {
    if (it.chunks > 1) ws.ml[place] = make_float2(mm, ll);
    else lse[me.hd] = mm == -INFINITY ? logf(ll) : mm + logf(ll);
  };
  // row 4 g4 + r of product (p, j) is dimension 64 p + 4 (4 g4 + r) + j
  if (!mine) return;
  const float inv = it.chunks > 1 ? 1.f : (l > 0.f ? 1.f / l : l);
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *(float4*)(to + 64 * p + 4 * (4 * g4 + r)) = make_float4(o[p][0][r] * inv, o[p][1][r] * inv, o[p][2][r] * inv, o[p][3][r] * inv);
  if (g4 == 0) sums(m, l);
}

// The chunks' states of (sequence, head) rows: a lane for four dims, `over` (a power of two) groups
// of such lanes over the chunks of a row, every lane's loads in flight together.
template <int D, bool BF>
__global__ __launch_bounds__(SH_T) void k_shared_join(SharedDims sd, int R, int places, int over, const int32_t* __restrict__ cu,
                                                      SharedWs ws, float* __restrict__ out, float* __restrict__ lse) {
  constexpr int LH = D / 4, GR = SH_T / LH, UN = 4;
  __shared__ float sM[GR], sS[GR];
  __shared__ __align__(16) float sO[GR][D];
  const int group = threadIdx.x / LH, gr = group & (over - 1), c = 4 * (threadIdx.x % LH);
  const int64_t hd = (int64_t)blockIdx.x * (GR / over) + group / over, rows = (int64_t)sd.n_seq * sd.H;
  const int64_t at = hd < rows ? hd : rows - 1;
  const int seq = (int)((uint32_t)at / (uint32_t)sd.H);
  const int b = sd.n_group > 1 ? span_with(cu, sd.n_group, seq) : 0;
  const Span sp = span_of(cu, b, sd.n_seq);
  bool on = hd < rows && seq >= sp.a && seq < sp.a + sp.n;      // in a group?
  const int4 x = ws.info[at];                                    // first chunk's place, chunks, places from one to the next, row there
  const int first = x.x, tiles = x.z, r = x.w & (R - 1);
  int chunks = x.y < places ? x.y : places;
  on &= chunks > 1;                                              // one: written already
  if (!on) chunks = 0;
  float M = -INFINITY, S = 0.f, O[4] = {0.f, 0.f, 0.f, 0.f};
  // a state of no entry has the maximum -inf and adds nothing, unless its sum is no number
  auto add = [&](float m, float s, const float4& x) {
    const float mn = fmaxf(M, m);
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((M - mn) * LOG2E);
    const float h = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * LOG2E);
    S = (f == 0.f && S == S ? 0.f : S * f) + (h == 0.f && s == s ? 0.f : s * h);
    const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i] = (f == 0.f ? 0.f : O[i] * f) + (h == 0.f ? 0.f : v[i] * h);
    M = mn;
  };
  // chunk p of the row's tile left its state at place first + p * tiles (where groups descend, that may be none)
  for (int p0 = gr; p0 < chunks; p0 += over * UN) {
    float2 ml[UN];
    float4 x[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int p = p0 + i * over < chunks ? p0 + i * over : p0;
      int64_t id = first + (int64_t)p * tiles;
      id = id < 0 ? 0 : (id >= places ? places - 1 : id);
      ml[i] = ws.ml[id * R + r];
      x[i] = *(const float4*)(ws.o + (id * R + r) * D + c);
    }
#pragma unroll
    for (int i = 0; i < UN; ++i)
      if (p0 + i * over < chunks) add(ml[i].x, ml[i].y, x[i]);
  }
  if (over > 1) {
    *(float4*)&sO[group][c] = make_float4(O[0], O[1], O[2], O[3]);
    if (c == 0) { sM[group] = M; sS[group] = S; }
    sync_after_lds_stores();
  }
  if (gr != 0 || !on) return;
  for (int i = 1; i < over; ++i) add(sM[group + i], sS[group + i], *(const float4*)&sO[group + i][c]);
  const float inv = S > 0.f ? 1.f / S : S;
  *(float4*)(out + at * D + c) = make_float4(O[0] * inv, O[1] * inv, O[2] * inv, O[3] * inv);
  if (c == 0) lse[at] = M == -INFINITY ? logf(S) : BF ? (M - SH_LAG * LN2) + logf(S * SH_TOP) : M + logf(S);
}

hipError_t launch_shared(const SharedDims& sd, const void* q, const int32_t* cu, const PrefixView& px, float* out, float* lse, void* base,
                         hipStream_t st) {
  const SharedPlan p = shared_plan(sd, px.rows);
  const SharedWs ws = shared_view(base, sd, p);
  const int room = p.places - (int)p.tiles;
  const dim3 grid((unsigned)p.places);
  const bool bf = sd.dtype == GRACEKV_BF16;
#define GKV_SHARED(TT, ...) hipLaunchKernelGGL((__VA_ARGS__), grid, dim3(64 * p.waves), 0, st, sd, room, (const TT*)q, cu, px, out, lse, ws)
  if (p.few) {
    if (bf) {
      if (sd.d == 64) GKV_SHARED(uint16_t, k_shared_few<uint16_t, 64, 2, 4>);
      else if (p.waves == 8) GKV_SHARED(uint16_t, k_shared_few<uint16_t, 128, 2, 8>);
      else GKV_SHARED(uint16_t, k_shared_few<uint16_t, 128, 2, 4>);
    } else {
      if (sd.d == 64) GKV_SHARED(float, k_shared_few<float, 64, 2, 4>);
      else if (p.waves == 8) GKV_SHARED(float, k_shared_few<float, 128, 1, 8>);
      else GKV_SHARED(float, k_shared_few<float, 128, 1, 4>);
    }
  } else if (bf) {
    if (sd.d == 128) {
      if (p.waves == 8) GKV_SHARED(uint16_t, k_shared_bf<128, 8>); else GKV_SHARED(uint16_t, k_shared_bf<128, 4>);
    } else {
      if (p.waves == 8) GKV_SHARED(uint16_t, k_shared_bf<64, 8>); else GKV_SHARED(uint16_t, k_shared_bf<64, 4>);
    }
  } else {
    if (sd.d == 128) GKV_SHARED(float, k_shared_f32<128>); else GKV_SHARED(float, k_shared_f32<64>);
  }
#undef GKV_SHARED
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.few) return e;
  auto join = [&](auto dim, auto bf16) {
    constexpr int D = decltype(dim)::value, GR = SH_T / (D / 4);
    const int chunks = room / (int)p.tiles;
    int over = 1;                        // about four chunks a lane, as it has loads in flight
    while (over < GR && over * 4 < chunks) over *= 2;
    const int64_t rows = (int64_t)sd.n_seq * sd.H, each = GR / over;
    hipLaunchKernelGGL((k_shared_join<D, decltype(bf16)::value>), dim3((unsigned)((rows + each - 1) / each)), dim3(SH_T), 0, st, sd, p.rows,
                       p.places, over, cu, ws, out, lse);
  };
  using std::integral_constant;
  if (bf) {
    if (sd.d == 128) join(integral_constant<int, 128>{}, std::true_type{}); else join(integral_constant<int, 64>{}, std::true_type{});
  } else {
    if (sd.d == 128) join(integral_constant<int, 128>{}, std::false_type{}); else join(integral_constant<int, 64>{}, std::false_type{});
  }
  return hipGetLastError();
}

}  // namespace gkv
