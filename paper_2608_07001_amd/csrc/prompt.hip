// Causal attention over packed prompts with grouped query heads.
//
// Sequence b has query rows [cu_q[b], cu_q[b+1]) and key rows [cu_k[b], cu_k[b+1]); its
// last query stands at its last key, so query i sees the keys j <= i + Lk - Lq:
//   out_i = sum_j softmax_j(q_i.k_j / sqrt(d)) v_j,  lse_i = log sum_j exp(q_i.k_j / sqrt(d))
// (no key: 0 and -inf).
//
// The query heads of a group share their keys, so the rows of a tile are (token, head)
// pairs, row r = token * hpg + head: any grouping fills the tile, keys and values are
// loaded once for the group, and the tile spans few tokens, which leaves little work
// above the diagonal.
//
// One pass over the keys with a running maximum and sum.  Products are formed transposed:
// S^T = K Q^T (keys x rows), then O^T = V^T P^T, because the accumulator of the first
// holds four neighbouring keys of one row per lane, which (the order of the keys inside a
// product is free) is the operand of the second: probabilities stay in their lane, and
// the row's maximum, sum and rescaling are lane-local but for one swap of halves.  Keys
// and values go through LDS, V^T by the transposing LDS read.
//
// A tile that some row of the workgroup sees in part (its diagonal, its end) is staged
// with values that are not finite replaced by 0, since 0 times an infinity is not 0; rows
// that do see such a value get it at the end.
//
// bf16 probabilities are rounded to bf16 (nearest even) as operands, their sum takes them
// unrounded: each weight is off by at most 2^-8 of itself, at random, like the output's
// own rounding, and the error against 64 bits is 0.5 to 3 % larger than that rounding's
// alone.  (A second part of the weights, as over pages, would add half of the products, which
// are what bounds long prompts.)  fp32 uses the fp32 matrix instructions.
//
// What bounds it: long prompts by the products and what goes on beside them.  16K tokens of
// the 8B heads take 1.97 to 2.03 ms on different devices, 1.09 to 1.13 PFLOP/s of the pairs
// that are seen (a library product of 8192^3 reaches 1.32): the matrix pipes are busy in
// 63 % of the cycles, LDS in 32 %, without a bank conflict, and the chip runs at 1.7 GHz of
// its 2.4; without the softmax, for timing, the same loop reached 1.26, without loads as
// well 1.36.  What was tried and left: tiles of
// 64 keys with two waves a SIMD (2.00 ms), through registers instead of straight into LDS
// (2.34), the two waves of a SIMD held in opposite phases by barriers (2.11 to 2.34), other
// orders and priorities of reads and products (within 1 %).  Short prompts and pieces are
// bound by the way along the keys, about 0.9 us a tile for a workgroup with few beside it
// (Plan), and by the parts' states, 33 MB of them for 64 queries over 32K keys: 50 us of
// products, 10 of joining.  fp32: 2048 tokens of the 8B heads 325 us, 106 TFLOP/s of 153.
#include "tiles.h"

namespace gkv {

constexpr int PR_T = 256;
constexpr int PR_W = PR_T / 64;
constexpr int PR_FILL = 512;       // workgroups that the keys of few rows are split into
constexpr int CUS = 256;
constexpr float PR_LAG = 8.f;      // base-2 units, and as a factor
constexpr float PR_TOP = 256.f;
constexpr float LOG2E = 1.44269504088896341f, LN2 = 0.693147180559945309f;

static size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

// Rows and keys of a workgroup's tile: SPLIT of its waves have the same rows, with 32 keys
// each of a key tile (bf16: 32 rows a wave; fp32: 16)
template <bool BF, int SPLIT> constexpr int tile_rows() { return (BF ? 32 : 16) * PR_W / SPLIT; }
template <int SPLIT> constexpr int tile_keys() { return 32 * SPLIT; }

// Row tiles of all sequences: sequence b's begin at cu_q[b] * hpg / rows + b, which
// leaves each at least as many as it needs whatever the lengths are; one sequence alone
// has as many as all rows need.
GKV_HD int row_tiles(const PromptDims& pd, int rows) {
  const uint32_t n = (uint32_t)(pd.n_q * pd.hpg);
  return pd.n_seq > 1 ? (int)(n / rows) + pd.n_seq : (int)((n + rows - 1) / rows);
}

// The kernel and the parts that every row tile's keys are cut into.
struct Plan {
  bool split;                  // waves share rows
  int rows, parts;
};
static Plan prompt_plan(const PromptDims& pd) {
  const bool bf = pd.dtype == GRACEKV_BF16;
  auto tiles = [&](int rows) { return (int64_t)row_tiles(pd, rows) * pd.G; };
  constexpr int ROWS = tile_rows<true, 1>(), FEW = tile_rows<true, 2>();
  Plan p;
  // Prompts that leave the chip part empty are bound by the way along the keys, which waves
  // in pairs halve, as long as the tiles of 64 rows are not too few to be cut no further, and
  // the keys of the longest sequence (of n_seq, taken as twice the mean or all there are) not
  // so many that a long way is walked faster in parts.  The 8B heads, single (in parts) and
  // paired: 256 tokens 12.4 and 11.5 us, 512 18.6 and 15.9, 1024 28.1 and 25.9, 1536 44.8 and
  // 41.8, 2048 55 and 63; one KV head with 8 heads of 128, 3000 tokens 47.9 and 51.2, with 16
  // heads of 64, 3500 tokens 56 and 43; 2 with 8 of 128, three sequences of 3300 tokens 41.9
  // and 33.1; 64 queries over 32K keys 62.7 and 73.4; fewer tiles than PR_FILL / 2: 16 heads
  // of 128 on 4, 700 tokens 22.2 and 18.1, 64 heads of 64 on 8, 128 queries over 4000 keys
  // 24.7 and 42.0.
  const int64_t longest = 2 * pd.n_k / (pd.n_seq + 1);
  p.split = bf && tiles(FEW) >= (longest <= 1024 ? PR_FILL / 4 : PR_FILL / 2) && tiles(ROWS) < (pd.d == 128 ? PR_FILL : 2 * PR_FILL) &&
            longest <= (pd.d == 128 ? 2048 : 4096);
  p.rows = bf ? (p.split ? FEW : ROWS) : tile_rows<false, 1>();
  // One part where the tiles fill the chip (bf16: twice over; fp32, whose key tiles take
  // four times as long: three times, 1056 tokens of the 8B heads 134 -> 111 us; the same in
  // bf16 slows 1024 tokens down, 27 -> 39), more where they are few, each part holding at
  // least so many keys of the longest row that joining it is worth it (bf16 with 128: 256
  // tokens 12 -> 17 us; fp32 with 256: 300 tokens 27 -> 30).  The lengths lie on the device, so
  // one number of parts serves all sequences, and the longest row is taken to see all n_k keys,
  // as it does where one sequence holds most of them.  Batches of pieces as long as each other
  // are cut a little more often than they need: 31 x 16 queries over 256 keys (2 KV heads, 16
  // heads) 12.7 us and 12.8 uncut, 8 x 100 over 700 (4, 16) 26.0 and 24.5, 20 x 30 over 1000
  // (2, 8) 23.3 and 30.8, fp32 16 x 64 over 512 (8, 32) 118 and 120; with the longest estimated
  // as above the same.  Batches of very different ones are cut too little, since the row tiles
  // of the short count too: one query over 30000 keys of the 8B heads 32 us alone, 179 beside 15
  // over 50 (676 uncut); 64 over 32K 65 alone, 269 beside 7 x 64 over 200.
  const int64_t n = tiles(p.rows), fill = bf ? PR_FILL : PR_FILL + PR_FILL / 2, keys = bf ? 256 : 128;
  const int64_t want = n && !p.split ? (fill + n - 1) / n : 1, most = (pd.n_k + keys - 1) / keys;
  const int64_t cap = want > most ? (most < 1 ? 1 : most) : want;
  // ... and only where that pays, by what was measured, in us: a key tile's step on the longest
  // way (longer where workgroups share a CU), the second kernel, and the states, written and
  // read.  The 8B heads: 512 tokens 26 in two parts, 19 in one, 128 queries over 4096 keys 31 in 16, 27 in eight.
  const double join = 5, state = 2.0 * pd.n_q * pd.H * (4 * pd.d + 8) / 3.5e6;
  auto cost = [&](int64_t parts) {
    const double step = bf ? (n * parts > CUS ? 0.9 : 0.75) : (pd.d == 128 ? 2.2 : 1.2);
    return pd.n_k / 32.0 / parts * step + (parts > 1 ? state * parts + join : 0);
  };
  const int64_t even = (int64_t)sqrt(pd.n_k / 32.0 * (bf ? 0.9 : pd.d == 128 ? 2.2 : 1.2) / (state > 0 ? state : 1e-9) + 0.5);
  p.parts = 1;
  for (const int64_t x : {cap, even, even + 1, n ? CUS / n : 1, n ? 2 * CUS / n : 1})
    if (x > 1 && x <= cap && cost(x) < cost(p.parts)) p.parts = (int)x;
  return p;
}
int64_t prompt_items(const PromptDims& pd) {
  const Plan p = prompt_plan(pd);
  return (int64_t)row_tiles(pd, p.rows) * p.parts * pd.G;
}
size_t prompt_ws_bytes(const PromptDims& pd) {
  const int P = prompt_plan(pd).parts;
  if (P == 1) return 0;
  const size_t n = (size_t)P * pd.n_q * pd.H;
  return al256(n * 8) + n * pd.d * 4;
}

// what a workgroup works on (rows of all heads of a group, and keys, are below 2^31)
struct Item {
  int b, g, part;
  int q0, lq, k0, lk;          // the sequence's rows
  int r0, rows;                // first (token, head) row of the tile; rows of the sequence
  int t0, t1;                  // key tiles [t0, t1)
};

// The item of workgroup blockIdx.x; false where there is none.  Pairs of one KV head and
// part are neighbours modulo G, so with G a multiple of 8 a KV head stays on one XCD's
// L2.  Row tiles are taken from the last to the first, so a sequence's tiles with the most
// keys come first, and the last sequence's before the others'.  Where the tiles are few, a long
// sequence at the batch's beginning ends later for that: 4000 tokens and 11 x 200 of the 8B
// heads 168 us with the long one first, 150 with it last (the 70B heads' eight sequences of 1 to
// 4099 tokens take 354 to 357 in any order).  Sequences ordered by their lengths on the device
// gained 10 % there and cost 64 sequences of 64 tokens 26 -> 34 us.
template <int ROWS, int KEYS>
__device__ __forceinline__ bool find_item(const PromptDims& pd, const int32_t* cu_q, const int32_t* cu_k, int parts, Item& it) {
  uint32_t bid = blockIdx.x;
  it.g = (int)(bid % (uint32_t)pd.G);
  bid /= (uint32_t)pd.G;
  it.part = parts > 1 ? (int)(bid % (uint32_t)parts) : 0;
  if (parts > 1) bid /= (uint32_t)parts;
  const int slot = row_tiles(pd, ROWS) - 1 - (int)bid;
  auto first = [&](int b) { return (int)((uint32_t)(held((int64_t)cu_q[b], pd.n_q) * pd.hpg) / ROWS) + b; };
  it.b = pd.n_seq > 1 ? find_last(pd.n_seq, [&](int b) { return first(b) <= slot; }) : 0;
  const Span sq = span_of(cu_q, it.b, pd.n_q), sk = span_of(cu_k, it.b, pd.n_k);
  it.q0 = (int)sq.a; it.lq = (int)sq.n; it.k0 = (int)sk.a; it.lk = (int)sk.n;
  it.rows = it.lq * pd.hpg;
  const int tile = pd.n_seq > 1 ? slot - first(it.b) : slot;
  if (tile < 0 || tile >= (int)(((uint32_t)it.rows + ROWS - 1) / ROWS)) return false;
  it.r0 = tile * ROWS;
  // keys that the tile's last row sees
  const uint32_t last = (uint32_t)(it.rows - it.r0 > ROWS ? it.r0 + ROWS : it.rows) - 1;
  int n = (int)(last / (uint32_t)pd.hpg) + 1 + (it.lk - it.lq);
  n = n < 0 ? 0 : n;
  const int tiles = n / KEYS + (n % KEYS != 0);
  it.t0 = 0;
  it.t1 = tiles;
  if (parts > 1) {                     // the first tiles % parts of them take one more
    const int each = tiles / parts, more = tiles % parts;
    it.t0 = it.part * each + min(it.part, more);
    it.t1 = it.t0 + each + (it.part < more);
  }
  return true;
}

// bf16 pairs / floats with what is not finite replaced by 0; `any` says whether there was
__device__ __forceinline__ uint32_t finite_bf(uint32_t x, bool& any) {
  const bool h = (x & 0x7f800000u) == 0x7f800000u, l = (x & 0x7f80u) == 0x7f80u;
  any |= h | l;
  return (h ? 0u : x & 0xffff0000u) | (l ? 0u : x & 0xffffu);
}
__device__ __forceinline__ uint32_t finite_f(uint32_t x, bool& any) {
  const bool b = (x & 0x7f800000u) == 0x7f800000u;
  any |= b;
  return b ? 0u : x;
}
template <bool BF> __device__ __forceinline__ uint4 finite(uint4 x, bool& any) {
  if constexpr (BF) return make_uint4(finite_bf(x.x, any), finite_bf(x.y, any), finite_bf(x.z, any), finite_bf(x.w, any));
  else return make_uint4(finite_f(x.x, any), finite_f(x.y, any), finite_f(x.z, any), finite_f(x.w, any));
}

template <int D, int SPLIT>
__global__ __launch_bounds__(PR_T, SPLIT == 2 && D == 128 ? 2 : 3) void k_prompt_bf(PromptDims pd, int parts, const uint16_t* __restrict__ q,
                                                       const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                       const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k,
                                                       uint16_t* __restrict__ out, float* __restrict__ lse,
                                                       float2* __restrict__ pml, float* __restrict__ po) {
  constexpr int ROWS = tile_rows<true, SPLIT>(), KEYS = tile_keys<SPLIT>();
  // Pairs form the next tile's logits beside the present one's softmax, which their LDS, two
  // workgroups a CU, leaves registers for: 1024 tokens of the 8B heads 27.6 -> 25.6 us, 1536
  // 44.8 -> 41.5.  Single waves gain nothing (2048 tokens 57.4 -> 60.8) and lose the third (16K
  // 2.08 -> 2.22 ms).
  constexpr bool AHEAD = SPLIT == 2 && D == 128;
  constexpr int CH = D / 8;                     // 16-byte pieces of a row
  constexpr int RI = 64 / CH;                   // rows that one load of a wave brings
  constexpr int NI = KEYS / RI / PR_W;          // such loads of a wave and array
  constexpr int KS = D / 16;                    // product steps over the dims
  constexpr int DT = D / 32;                    // 32-dim tiles of the output
  // arrays of their own, so that loads into one tile and reads of the other are told apart
  __shared__ __align__(16) uint4 sK0[KEYS * CH], sK1[KEYS * CH], sV0[KEYS * CH], sV1[KEYS * CH];
  __shared__ int bad;
  Item it;
  if (!find_item<ROWS, KEYS>(pd, cu_q, cu_k, parts, it)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i32 = lane & 31, half = lane >> 5;
  const int rw = w / SPLIT, kw = w % SPLIT;     // the wave's 32 rows, its 32 keys of a tile
  const int off = it.lk - it.lq;                // query i sees the keys up to i + off
  // the lane's row
  const uint32_t hpg = (uint32_t)pd.hpg;
  const int row = it.r0 + 32 * rw + i32, rowc = row < it.rows ? row : it.rows - 1;
  const int tok = (int)((uint32_t)rowc / hpg);
  const int head = it.g * pd.hpg + (rowc - tok * pd.hpg);
  const int see = tok + off;                    // its last key
  // what the wave's and the workgroup's rows see
  const int wr0 = it.r0 + 32 * rw, wr1 = min(wr0 + 31, it.rows - 1);
  const int w_all = (int)((uint32_t)min(wr0, it.rows - 1) / hpg) + off;
  const int w_any = wr0 < it.rows ? (int)((uint32_t)wr1 / hpg) + off : -1;
  const int g_all = (int)((uint32_t)it.r0 / hpg) + off;

  uint4 qv[KS];
  {
    const uint16_t* qp = q + (int64_t)(it.q0 + tok) * pd.q_tok + head * pd.q_head;
#pragma unroll
    for (int s = 0; s < KS; ++s) qv[s] = *(const uint4*)(qp + 16 * s + 8 * half);
  }
  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[t][r] = 0.f;
  float m = -INFINITY, l = 0.f;                 // what is subtracted, base-2 units; l: this lane's keys only
  const float sc2 = LOG2E / sqrtf((float)D);

  const uint16_t* kp = k + it.k0 * pd.k_tok + it.g * pd.k_head;
  const uint16_t* vp = v + it.k0 * pd.v_tok + it.g * pd.v_head;
  // Load i of a wave brings rows RI (w + PR_W i) .. + RI - 1 straight into LDS, lane l to
  // the l-th 16 bytes: the piece that swz() puts there
  const int lr = RI * w + lane / CH, lc = swz<D>(lr, lane % CH) - lr * CH;
  const int k_off = (int)(lr * pd.k_tok * 2) + lc * 16, k_step = (int)(RI * PR_W * pd.k_tok * 2);
  const int v_off = (int)(lr * pd.v_tok * 2) + lc * 16, v_step = (int)(RI * PR_W * pd.v_tok * 2);
  auto load = [&](const uint16_t* rows, int64_t stride, int off, int by, int t, uint4* to) {
    const int n = min(it.lk - t * KEYS, KEYS);   // at least one
    const Buffer b = tile_buffer<uint16_t, D>(rows + (int64_t)t * KEYS * stride, stride, n);
#pragma unroll
    for (int i = 0; i < NI; ++i) buffer_load_lds(b, to + 64 * (w + PR_W * i), off + i * by);
  };
  auto load_keys = [&](int t, uint4* to) { load(kp, pd.k_tok, k_off, k_step, t, to); };
  auto load_values = [&](int t, uint4* to) { load(vp, pd.v_tok, v_off, v_step, t, to); };
  // Where the lane reads in a tile, in bytes: piece 2 x + half of key row i32 lies at
  // k_at ^ 32 x; row 4 half + (lane % 16) / 4 of the transposing read's 8 bytes at v_at,
  // dim tile d at v_at ^ 64 d, the row 8 further at ^ 32 (swz()).
  constexpr int RB = 2 * D;
  int k_at = 16 * swz<D>(i32, half);
  const int v_at = 16 * swz<D>(4 * half + ((lane & 15) >> 2), 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) + 8 * (lane & 1);
  auto logits = [&](const uint4* cK) __attribute__((always_inline)) {
    f32x16 s;
    asm volatile("" : "+v"(k_at));               // eight places: formed anew, not held in registers
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int x = 0; x < KS; ++x) s = mfma_bf16_32x32x16(lds_at(cK, (k_at ^ (32 * x)) + 32 * kw * RB), qv[x], s);
    return s;
  };
  f32x16 s;                                      // AHEAD: the logits of the tile whose turn it is
  auto step = [&](int t, uint4* cK, uint4* cV, uint4* nK, uint4* nV) __attribute__((always_inline)) {
    // the wave's own loads of tile t are there, then everyone's; and everyone is done with
    // tile t - 1, which t + 1 replaces.  (A third tile in flight was slower for long prompts:
    // 16K 1985 -> 2014 us, 8K 522 -> 536, though not for a ragged batch, 367 -> 360.)
    wait_vm();
    sync_after_lds_stores();
    const int j0 = t * KEYS;
    if (j0 + (KEYS - 1) > g_all) {              // values that are not finite: see above
      bool any = false;
#pragma unroll
      for (int i = 0; i < KEYS * CH / PR_T; ++i) cV[tid + PR_T * i] = finite<true>(cV[tid + PR_T * i], any);
      if (any) bad = 1;
      sync_after_lds_stores();
    }
    if constexpr (AHEAD) {
      if (t + 2 < it.t1) load_keys(t + 2, cK);   // whose keys are logits already
      if (t + 1 < it.t1) load_values(t + 1, nV);
    } else if (t + 1 < it.t1) {
      load_keys(t + 1, nK);
      load_values(t + 1, nV);
    }
    const int k0 = j0 + 32 * kw;                 // the wave's keys
    if (k0 > w_any) return;
    if constexpr (!AHEAD) {
      s = logits(cK);
      reads_ahead<KS, 1, 4>();
    }
    mfma_done16(s);
    // register r: key 8 (r / 4) + 4 half + r % 4
    if (k0 + 31 > w_all) {
      const int rel = see - k0 - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 8 * (r / 4) + r % 4 > rel ? -INFINITY : s[r];
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    {
      const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1])) * sc2;
    }
    // What is subtracted stands PR_LAG above a maximum that may lag behind by as much: the outputs
    // are rescaled seldom, no weight is above 1 (sums of large values stay in range as under the
    // maximum itself), the row's largest at least 2^-PR_LAG, and all are as exact
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx + PR_LAG);
      const float c = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= c;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= c;
    }
    const float ms = m == -INFINITY ? 0.f : m;
    f32x16 sn;
    if constexpr (AHEAD) {                       // past the last tile: of what is there, and not used
      sn = logits(nK);
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int x = 0; x < KS; ++x) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (x + 4 < KS) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x002, 72 / KS, 0);      // vector instructions
      }
    }
    uint4 pr[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      float e[8];
#pragma unroll
      for (int r = 0; r < 8; ++r) e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[8 * h + r], sc2, -ms));
      l += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      pr[h] = make_uint4(pack_bf16(e[0], e[1]), pack_bf16(e[2], e[3]), pack_bf16(e[4], e[5]), pack_bf16(e[6], e[7]));
    }
    // product step x: keys 16 x + 8 (j / 4) + 4 half + j % 4 in place 8 half + j
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const uint2 a = lds_read_tr(cV, (v_at ^ (64 * d)) + (32 * kw + 16 * x) * RB);
        const uint2 b = lds_read_tr(cV, (v_at ^ (64 * d + 32)) + (32 * kw + 16 * x + 8) * RB);
        o[d] = mfma_bf16_32x32x16(make_uint4(a.x, a.y, b.x, b.y), pr[x], o[d]);
      }
    reads_ahead<2 * DT, 2, 3>();
    if constexpr (AHEAD) s = sn;
  };
  if (tid == 0) bad = 0;
  if (it.t0 < it.t1) {
    load_keys(it.t0, sK0);
    load_values(it.t0, sV0);
    if constexpr (AHEAD) {
      if (it.t0 + 1 < it.t1) load_keys(it.t0 + 1, sK1);
      wait_vm();
      sync_after_lds_stores();
      s = logits(sK0);
    }
  }
  for (int t = it.t0; t < it.t1; t += 2) {
    step(t, sK0, sV0, sK1, sV1);
    if (t + 1 < it.t1) step(t + 1, sK1, sV1, sK0, sV0);
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) mfma_done16(o[d]);
  sync_after_lds_stores();
  if constexpr (SPLIT == 2) {                   // the second wave of a pair to the first, through the tiles' LDS
    static_assert(PR_W / SPLIT == 2 && KEYS * CH * 16 >= 64 * 4 * 16 * DT, "an array for each pair");
    __shared__ float2 sml[PR_W / SPLIT][64];
    float* so = (float*)(rw == 0 ? sK0 : sK1);
    if (kw == 1) {
      sml[rw][lane] = make_float2(m, l);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) so[64 * (16 * d + r) + lane] = o[d][r];
    }
    sync_after_lds_stores();
    if (kw == 1) return;
    const float2 x = sml[rw][lane];
    const float mn = fmaxf(m, x.x);
    const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn), g = x.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x.x - mn);
    l = (f == 0.f && l == l ? 0.f : l * f) + (g == 0.f && x.y == x.y ? 0.f : x.y * g);       // NaN stays
    m = mn;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float y = so[64 * (16 * d + r) + lane];
        o[d][r] = (f == 0.f ? 0.f : o[d][r] * f) + (g == 0.f ? 0.f : y * g);
      }
  }
  // values that are not finite in partly seen tiles, for the rows that see them
  if (bad) {
    for (int j = max(max(g_all + 1, 0) / KEYS, it.t0) * KEYS; j < min(it.t1 * KEYS, it.lk); ++j)
      if (j <= see) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float x = bf16_to_f32(vp[(int64_t)j * pd.v_tok + 32 * d + 8 * (r / 4) + 4 * half + r % 4]);
            if (!(fabsf(x) < INFINITY)) o[d][r] += x;
          }
      }
  }
  {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  }
  if (row >= it.rows) return;
  const int64_t qrow = (int64_t)it.q0 + tok;
  if (parts > 1) {
    const int64_t part = ((int64_t)it.part * pd.n_q + qrow) * pd.H + head;
    if (half == 0) pml[part] = make_float2(m, l);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *(float4*)(po + part * D + 32 * d + 8 * r + 4 * half) = make_float4(o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]);
    return;
  }
  const float inv = l > 0.f ? 1.f / l : l;      // no key: the sums are 0; NaN stays
  uint16_t* op = out + qrow * pd.o_tok + head * pd.o_head;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *(uint2*)(op + 32 * d + 8 * r + 4 * half) =
          make_uint2(pack_bf16(o[d][4 * r] * inv, o[d][4 * r + 1] * inv), pack_bf16(o[d][4 * r + 2] * inv, o[d][4 * r + 3] * inv));
  // (with the sum in units of its largest weight, whose logarithm is small)
  if (lse && half == 0) lse[qrow * pd.H + head] = m == -INFINITY ? logf(l) : ((m - PR_LAG) + log2f(l * PR_TOP)) * LN2;
}

// fp32: 16 rows a wave, 32 keys a tile, fp32 matrix instructions
template <int D>
__global__ __launch_bounds__(PR_T, 2) void k_prompt_f32(PromptDims pd, int parts, const float* __restrict__ q,
                                                        const float* __restrict__ k, const float* __restrict__ v,
                                                        const int32_t* __restrict__ cu_q, const int32_t* __restrict__ cu_k,
                                                        float* __restrict__ out, float* __restrict__ lse,
                                                        float2* __restrict__ pml, float* __restrict__ po) {
  constexpr int ROWS = tile_rows<false, 1>(), KEYS = tile_keys<1>();
  constexpr int CH = D / 4, NL = KEYS * CH / PR_T, LD = D + 4;
  constexpr int KC = D / 16, VB = D / 64;
  __shared__ __align__(16) float sK[KEYS * LD], sV[KEYS * LD];
  __shared__ int bad;
  Item it;
  if (!find_item<ROWS, KEYS>(pd, cu_q, cu_k, parts, it)) return;
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, i16 = lane & 15, g4 = lane >> 4;
  const uint32_t hpg = (uint32_t)pd.hpg;
  const int off = it.lk - it.lq;
  const int row = it.r0 + 16 * w + i16, rowc = row < it.rows ? row : it.rows - 1;
  const int tok = (int)((uint32_t)rowc / hpg);
  const int head = it.g * pd.hpg + (rowc - tok * pd.hpg);
  const int see = tok + off;
  const int wr0 = it.r0 + 16 * w, wr1 = min(wr0 + 15, it.rows - 1);
  const int w_any = wr0 < it.rows ? (int)((uint32_t)wr1 / hpg) + off : -1;
  const int g_all = (int)((uint32_t)it.r0 / hpg) + off;

  float4 qv[KC];                                // pieces g4, g4 + 4, ... of the row
  {
    const float* qp = q + (int64_t)(it.q0 + tok) * pd.q_tok + head * pd.q_head;
#pragma unroll
    for (int s = 0; s < KC; ++s) qv[s] = *(const float4*)(qp + 16 * s + 4 * g4);
  }
  f32x4 o[VB][4];
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int j = 0; j < 4; ++j) o[p][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;
  const float sc2 = LOG2E / sqrtf((float)D);
  const float* kp = k + it.k0 * pd.k_tok + it.g * pd.k_head;
  const float* vp = v + it.k0 * pd.v_tok + it.g * pd.v_head;
  uint4 rk[NL], rv[NL];
  auto load = [&](int t) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int e = tid + PR_T * i, c = e % CH;
      const int64_t j = (int64_t)t * KEYS + e / CH;
      const bool in = j < it.lk;
      rk[i] = in ? *(const uint4*)(kp + j * pd.k_tok + 4 * c) : make_uint4(0, 0, 0, 0);
      rv[i] = in ? *(const uint4*)(vp + j * pd.v_tok + 4 * c) : make_uint4(0, 0, 0, 0);
    }
  };
  if (tid == 0) bad = 0;
  if (it.t0 < it.t1) load(it.t0);
  for (int t = it.t0; t < it.t1; ++t) {
    sync_after_lds_stores();
    if (t * KEYS + (KEYS - 1) > g_all) {
      bool any = false;
#pragma unroll
      for (int i = 0; i < NL; ++i) rv[i] = finite<false>(rv[i], any);
      if (any) bad = 1;
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int e = tid + PR_T * i;
      *(uint4*)(sK + e / CH * LD + 4 * (e % CH)) = rk[i];
      *(uint4*)(sV + e / CH * LD + 4 * (e % CH)) = rv[i];
    }
    if (t + 1 < it.t1) load(t + 1);
    sync_after_lds_stores();
    const int j0 = t * KEYS;
    if (j0 > w_any) continue;
    float x[KEYS / 16][4];
#pragma unroll
    for (int b = 0; b < KEYS / 16; ++b) {
      f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KC; ++s) {
        const float4 a = *(const float4*)(sK + (16 * b + i16) * LD + 16 * s + 4 * g4);
        acc = mfma_f32_16x16x4(a.x, qv[s].x, acc);
        acc = mfma_f32_16x16x4(a.y, qv[s].y, acc);
        acc = mfma_f32_16x16x4(a.z, qv[s].z, acc);
        acc = mfma_f32_16x16x4(a.w, qv[s].w, acc);
      }
      mfma_done(acc);
#pragma unroll
      for (int r = 0; r < 4; ++r) x[b][r] = j0 + 16 * b + 4 * g4 + r > see ? -INFINITY : acc[r];
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
      mx = fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])) * sc2;
    }
    if (__any(mx > m)) {
      const float mn = fmaxf(m, mx);
      const float c = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
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
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][r], sc2, -ms));
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
  sync_after_lds_stores();
  // row 4 g4 + r of product (p, j) is dimension 64 p + 4 (4 g4 + r) + j
  if (bad) {
    for (int j = max(max(g_all + 1, 0) / KEYS, it.t0) * KEYS; j < min(it.t1 * KEYS, it.lk); ++j)
      if (j <= see) {
#pragma unroll
        for (int p = 0; p < VB; ++p)
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = vp[(int64_t)j * pd.v_tok + 64 * p + 4 * (4 * g4 + r) + i];
              if (!(fabsf(x) < INFINITY)) o[p][i][r] += x;
            }
      }
  }
  l = col_sum4(l);
  if (row >= it.rows) return;
  const int64_t qrow = (int64_t)it.q0 + tok;
  const int64_t part = ((int64_t)it.part * pd.n_q + qrow) * pd.H + head;
  const float inv = parts > 1 ? 1.f : (l > 0.f ? 1.f / l : l);
  float* op = parts > 1 ? po + part * D : out + qrow * pd.o_tok + head * pd.o_head;
#pragma unroll
  for (int p = 0; p < VB; ++p)
#pragma unroll
    for (int r = 0; r < 4; ++r)
      *(float4*)(op + 64 * p + 4 * (4 * g4 + r)) = make_float4(o[p][0][r] * inv, o[p][1][r] * inv, o[p][2][r] * inv, o[p][3][r] * inv);
  if (g4 != 0) return;
  if (parts > 1) pml[part] = make_float2(m, l);
  else if (lse) lse[qrow * pd.H + head] = m == -INFINITY ? logf(l) : (m + log2f(l)) * LN2;
}

// The parts of (token, head) rows: a lane for four dims, `over` (a power of two) groups of
// such lanes over the parts of a row, every lane's loads in flight together.
template <typename T, int D>
__global__ __launch_bounds__(PR_T) void k_prompt_combine(PromptDims pd, int parts, int over, const int32_t* __restrict__ cu_q,
                                                         const float2* __restrict__ pml, const float* __restrict__ po,
                                                         T* __restrict__ out, float* __restrict__ lse) {
  constexpr int LH = D / 4, GR = PR_T / LH, UN = 4;
  __shared__ float sM[GR], sS[GR];
  __shared__ __align__(16) float sO[GR][D];
  const int group = threadIdx.x / LH, gr = group & (over - 1), c = 4 * (threadIdx.x % LH);
  const int64_t row = (int64_t)blockIdx.x * (GR / over) + group / over, rows = pd.n_q * pd.H;
  const int64_t at = row < rows ? row : rows - 1;
  const int t = (int)((uint32_t)at / (uint32_t)pd.H), head = (int)at - t * pd.H;
  // is the token in a sequence?  (rows behind the last one are nobody's)
  const int b = pd.n_seq > 1 ? span_with(cu_q, pd.n_seq, t) : 0;
  const Span sp = span_of(cu_q, b, pd.n_q);
  const bool on = row < rows && t >= sp.a && t < sp.a + sp.n;
  const int64_t step = pd.n_q * pd.H;
  float M = -INFINITY, S = 0.f, O[4] = {0.f, 0.f, 0.f, 0.f};
  // a state of no key has the maximum -inf and adds nothing, unless its sum is no number
  auto add = [&](float m, float s, const float4& x) {
    const float mn = fmaxf(M, m);
    const float f = M == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(M - mn), g = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
    S = (f == 0.f && S == S ? 0.f : S * f) + (g == 0.f && s == s ? 0.f : s * g);
    const float v[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i] = (f == 0.f ? 0.f : O[i] * f) + (g == 0.f ? 0.f : v[i] * g);
    M = mn;
  };
  for (int p0 = gr; p0 < parts && on; p0 += over * UN) {
    float2 ml[UN];
    float4 x[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
      const int64_t p = at + (p0 + i * over < parts ? p0 + i * over : p0) * step;
      ml[i] = pml[p];
      x[i] = *(const float4*)(po + p * D + c);
    }
#pragma unroll
    for (int i = 0; i < UN; ++i)
      if (p0 + i * over < parts) add(ml[i].x, ml[i].y, x[i]);
  }
  if (over > 1) {
    *(float4*)&sO[group][c] = make_float4(O[0], O[1], O[2], O[3]);
    if (c == 0) { sM[group] = M; sS[group] = S; }
    sync_after_lds_stores();
  }
  if (gr != 0 || !on) return;
  for (int i = 1; i < over; ++i) add(sM[group + i], sS[group + i], *(const float4*)&sO[group + i][c]);
#pragma unroll
  for (int i = 0; i < 4; ++i) stf(out, t * pd.o_tok + head * pd.o_head + c + i, S > 0.f ? O[i] / S : S);
  if (lse && c == 0) lse[at] = M == -INFINITY ? logf(S) : (M + log2f(S)) * LN2;
}

hipError_t launch_prompt(const PromptDims& pd, const void* q, const void* k, const void* v, const int32_t* cu_q,
                         const int32_t* cu_k, void* out, float* lse, void* ws, hipStream_t st) {
  if (pd.n_q == 0) return hipSuccess;
  const Plan plan = prompt_plan(pd);
  const int P = plan.parts;
  float2* pml = P > 1 ? (float2*)ws : nullptr;
  float* po = P > 1 ? (float*)((char*)ws + al256((size_t)P * pd.n_q * pd.H * 8)) : nullptr;
  const bool bf = pd.dtype == GRACEKV_BF16;
  const dim3 grid((unsigned)prompt_items(pd));
#define GKV_PROMPT(TT, ...)                                                                                                  \
  hipLaunchKernelGGL((__VA_ARGS__), grid, dim3(PR_T), 0, st, pd, P, (const TT*)q, (const TT*)k, (const TT*)v, cu_q, cu_k, (TT*)out, \
                     lse, pml, po)
  if (bf) {
    if (plan.split) {
      if (pd.d == 128) GKV_PROMPT(uint16_t, k_prompt_bf<128, 2>); else GKV_PROMPT(uint16_t, k_prompt_bf<64, 2>);
    } else {
      if (pd.d == 128) GKV_PROMPT(uint16_t, k_prompt_bf<128, 1>); else GKV_PROMPT(uint16_t, k_prompt_bf<64, 1>);
    }
  } else {
    if (pd.d == 128) GKV_PROMPT(float, k_prompt_f32<128>); else GKV_PROMPT(float, k_prompt_f32<64>);
  }
#undef GKV_PROMPT
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || P == 1) return e;
  auto join = [&](auto type, auto dim) {
    using T = decltype(type);
    constexpr int D = decltype(dim)::value, GR = PR_T / (D / 4);
    int over = 1;                        // about four parts a lane, as it has loads in flight
    while (over < GR && over * 4 < P) over *= 2;
    const int64_t rows = pd.n_q * pd.H, each = GR / over;
    hipLaunchKernelGGL((k_prompt_combine<T, D>), dim3((unsigned)((rows + each - 1) / each)), dim3(PR_T), 0, st, pd, P, over, cu_q,
                       pml, po, (T*)out, lse);
  };
  using std::integral_constant;
  if (bf) {
    if (pd.d == 128) join(uint16_t{}, integral_constant<int, 128>{}); else join(uint16_t{}, integral_constant<int, 64>{});
  } else {
    if (pd.d == 128) join(float{}, integral_constant<int, 128>{}); else join(float{}, integral_constant<int, 64>{});
  }
  return hipGetLastError();
}

}  // namespace gkv
