// Where a token lies in a paged cache, which sequence a packed row belongs to, and how
// rows of a cache are cut into chunks: the index arithmetic of the append and paged
// attention kernels, plain C++ so that the host can run it as well.  Nothing here reads
// memory except through `cu`.
//
// A cache holds n_pages pages of `1 << shift` tokens, page_stride elements apart,
// each [G][1 << shift][d].  A sequence's row of the block table names its pages in
// order; a place whose id lies outside [0, n_pages) holds no page.
#pragma once

#include <math.h>
#include <stdint.h>

#ifdef __HIP_DEVICE_COMPILE__
#define GKV_HD __host__ __device__ __forceinline__
#elif defined(__HIPCC__)
#define GKV_HD __host__ __device__ inline
#else
#define GKV_HD inline
#endif

namespace gkv {

struct PageDims {
  int dtype, G, H, d, hpg, n_seq;
  int shift, width;             // log2 of the tokens of a page; page ids of a sequence
  int64_t n_pages, page_stride;
};

// element of (token `at` of page `id`, KV head g, dim 0), or -1 where there is no such page
GKV_HD int64_t page_row(const PageDims& p, int64_t id, int g, int at) {
  if (id < 0 || id >= p.n_pages) return -1;
  return id * p.page_stride + (((int64_t)g << p.shift) + at) * p.d;
}

// tokens of a sequence, held to what its row of the table can name
GKV_HD int64_t held_len(const PageDims& p, int64_t len) {
  const int64_t most = (int64_t)p.width << p.shift;
  return len < 0 ? 0 : (len > most ? most : len);
}

// bounds of sequence b in packed rows (n of them), as given by the n_seq + 1 ascending
// starts `cu`: held inside [0, n], and empty where this pair descends (which of several
// sequences a row belongs to is then not told: find_last, span_with)
struct Span { int64_t a, n; };
GKV_HD int64_t held(int64_t x, int64_t n) { return x < 0 ? 0 : (x > n ? n : x); }
GKV_HD Span span_of(const int32_t* cu, int b, int64_t n) {
  const int64_t a = held(cu[b], n), e = held(cu[b + 1], n);
  return {a, e < a ? 0 : e - a};
}

// ---- chunks of paged attention ----
constexpr int64_t PAGED_ROWS = 1 << 25;  // most tokens of a sequence's pages, and most packed entries of a row
constexpr int PA_T = 256;
constexpr int PA_W = PA_T / 64;
constexpr int PA_HEADS = 16;       // query heads of a workgroup
constexpr int PA_MIN = PA_W;       // tiles of the shortest chunk: one a wave
// Chunks that the rows are cut into: as many as the chip holds (three workgroups a CU) for
// few rows, twice that for many, whose own ends then even out.  Rows below PA_FEW count as
// few: 192 rows of compressed contexts 47.0 us with 768, 51.8 with 1536; 512 rows of ragged
// sequences 74.8 with 1024, 73.4 with 1536, 74.0 with 2048.
constexpr int PA_TARGET = 1536, PA_FEW = 256;
// Joining the states of a row's chunks against a tile's step (chunks_of; half or twice as much
// is up to a fifth slower).  Without that limit on the chunks of a row one sequence of 128K
// tokens and one KV head took 240 us with 16 query heads of 128 and 77 with one of 64; now 55
// and 24.
constexpr float PA_COST = 0.6f;
GKV_HD float join_cost(int hpg, int d) {
  return PA_COST * (((hpg < PA_HEADS ? hpg : PA_HEADS) * (d / 2) + PA_T - 1) / PA_T);    // by passes over the heads
}

// Tiles of a row.  It has at most PAGED_ROWS tokens in pages and as many packed entries: 2^22
// tiles, so that those of 256 rows are counted in 31 bits.
template <int TILE> GKV_HD int tiles_of(int64_t len, int64_t count) {
  const int t = (int)((len + TILE - 1) / TILE) + (int)((count + TILE - 1) / TILE);
  return t > 0 ? t : 1;              // an empty row has a chunk, which writes its zeros
}

// Places of the grid beside one a row: half the rows leave theirs unfilled, and no more than
// the shortest chunks of the longest rows could make.  The px_rows packed entries count once,
// as they do where every row has its own.  Rows that share them (a compressed context that
// many sequences begin with) are then cut less than others as long, which suits most: shared
// entries come from L2, and joining is not free.  64 sequences with 8 KV heads over 2048
// shared entries a head 50 us, 61 with the entries counted for every row; 200 with 4 over 1024
// 33 and 46; 4 with 8 over 2048 16.0 and 16.6; but 16 with 8 over 4096 36 and 31.
GKV_HD int64_t chunk_room(const PageDims& p, int64_t px_rows, int tile) {
  const int64_t R = (int64_t)p.n_seq * p.G;
  const int64_t tiles = R * ((((int64_t)p.width << p.shift) + tile - 1) / tile) + (px_rows ? px_rows / tile + R : 0);
  const int64_t room = (tiles + PA_MIN - 1) / PA_MIN;
  const int64_t target = R < PA_FEW ? PA_TARGET / 2 : PA_TARGET;
  const int64_t most = target - R / 2 > target / 4 ? target - R / 2 : target / 4;
  return room < 1 ? 1 : (room > most ? most : room);
}

// Tiles of a chunk: all rows' tiles over the places that the grid leaves beside one a row
// (every row may leave one chunk unfilled), and no fewer than the waves.
GKV_HD int chunk_tiles(uint64_t total, int room) {
  const uint64_t size = total < 0x7fffffffu ? ((uint32_t)total + (uint32_t)room - 1) / (uint32_t)room : (total + room - 1) / room;
  return size < (uint64_t)PA_MIN ? PA_MIN : (size > 0x7fffffffu ? 0x7fffffff : (int)size);
}
// ... and chunks of a row of n tiles (below 2^24), n / size upwards, where size is also no less
// than sqrt(join n), in whole steps of the waves.  A workgroup walks size / PA_W tiles a wave,
// one after the other, and the last of a row's joins n / size states, some at a time, in join's
// passes over the heads: the longer of few rows are bound by the sum of both.
GKV_HD int chunks_of(int n, int size, float join) {
  const int least = ((int)sqrtf(join * (float)n) + PA_W / 2) & ~(PA_W - 1);
  size = size < least ? least : size;
  int c = (int)((float)n * (1.0f / (float)size));      // or next to it
  int left = n - c * size;
  if (left < 0) { --c; left += size; }
  else if (left >= size) { ++c; left -= size; }
  return c + (left > 0);
}

// ---- quantised pages: eight waves a workgroup ----
constexpr int PA_CUS = 256;        // workgroups of eight waves that run at once (their registers)

// Eight waves for few rows that may be long: half the chunks, whose states the last joins in half the time
// (with more threads, which is what counts for many heads).  The lengths are not known here: what the table can name counts.
// us with four and eight, 8 KV heads of 128, bf16 over e4m3, ragged: from 1 to the longest:
//   32 query heads: one sequence of 2048 tokens 9.7, 9.9, of 8192 13.1, 12.8; 3 of 8192 20.6, 16.7; 8 of 8192 29.4, 28.3; 8 ragged to
//     4096 14.6, 12.7, to 8192 20.4, 18.4;  64 query heads: 512 10.4, 10.0; 8192 15.8, 13.2; 8 ragged to 8192 23.5, 18.5
//   fp32, 4 of 8192 26.6, 19.5; heads of 64, 4 of 8192 15.0, 13.0
// More than 64 rows (9 sequences) are seldom better and often worse, whether their chunks fit the chip or not: 16 ragged to
// 8192 33.9, 50 (38 where they fit), 20 ragged 37.0, 40 (53), 12 of 4096 23.2, 34 (24), 31 of 4096 47.2, 44.6; fp32, 16 ragged
// 45, 58 (46).  Of short ones with many heads, which make a chunk or two a row, they stay better: 64 query heads, 12 of 512 11.7, 10.3, 24 of
// 512 14.3, 10.2, 31 ragged to 768 14.4, 11.7 (20 of 1024 18.2, 23).  More than 16 heads a KV head are two workgroups a chunk: 100 of 768 23, 28.
inline bool eight_waves(const PageDims& p) {
  const int64_t R = (int64_t)p.n_seq * p.G, cap = (int64_t)p.width << p.shift;
  if (R > 64) return R < PA_CUS && p.hpg > 4 && p.hpg <= PA_HEADS && cap >= 512 && cap <= 768;
  return p.hpg > 4 ? cap >= 512 : R * cap >= 131072;
}
// Tiles of their chunks: where those of `size` tiles would be more than the chip runs at once, longer ones, which are no
// more (a few in a second round: 7 sequences of 32768 tokens 129 us for 90, 53 of 8192 of one KV head 38 for 25).
GKV_HD int one_round(uint64_t total, int rows, int size, int64_t chunks) {
  return chunks > PA_CUS ? chunk_tiles(total, PA_CUS - rows) : size;
}

}  // namespace gkv
