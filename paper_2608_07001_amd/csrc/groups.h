// How the rows of groups of sequences that share entries are tiled, and how their entries are
// cut into chunks: index arithmetic of shared.hip, plain C++ so that the host can run it as
// well.  Nothing here reads memory except through `cu`.
//
// A group's rows (sequence, query head of a KV head), row = sequence * hpg + head, fill row
// tiles of R rows; the group's entries of that KV head, n key tiles of them, are cut into
// chunks, and a workgroup takes one chunk for one row tile.
#pragma once

#include "pages.h"

namespace gkv {

struct SharedDims {
  int dtype, G, H, d, hpg, n_seq, n_group;
  int64_t q_tok;
};

// Row tiles of every KV head: those of group b, whose first sequence is `a`, begin at a * hpg / R + b,
// which leaves each at least as many as it needs whatever the groups are.
GKV_HD int first_tile(const SharedDims& sd, int a, int b, int R) { return (int)((uint32_t)(a * sd.hpg) / (uint32_t)R) + b; }
GKV_HD int64_t most_tiles(const SharedDims& sd, int R) {
  return sd.n_group > 1 ? (int64_t)sd.n_seq * sd.hpg / R + sd.n_group : ((int64_t)sd.n_seq * sd.hpg + R - 1) / R;
}
GKV_HD int tiles_of_group(const SharedDims& sd, int64_t n, int R) { return (int)((n * sd.hpg + R - 1) / R); }

// Key tiles of a chunk: all row tiles' key tiles over the places that the grid has beside
// one a row tile (each may leave a chunk unfilled), and no fewer than `least`.
GKV_HD int shared_chunk(uint64_t total, int room, int least) {
  const uint64_t size = (total + (uint64_t)room - 1) / (uint64_t)room;
  return size < (uint64_t)least ? least : (size > 0x7fffffff ? 0x7fffffff : (int)size);
}

// The item of workgroup `bid` of `places` (a multiple of 8), `all` items in order: neighbours go to one XCD,
// workgroups going round the eight.  -1: none.  Groups that descend can make more items than places, of which
// the last are left out: an item's number is its place in the workspace.
GKV_HD int item_of(int bid, int all, int places) {
  const int n = all < places ? all : places, per = (n + 7) / 8, at = bid >> 3, id = (bid & 7) * per + at;
  return at < per && id < n ? id : -1;
}

constexpr int SH_T = 256;
constexpr int SH_W = SH_T / 64;
struct SharedPlan {
  bool few;                    // 16 rows a workgroup, its waves a tile of keys each
  int waves, rows, places;     // of a workgroup; rows of a tile; workgroups, a multiple of 8
  int64_t tiles;               // row tiles of all KV heads, at most
};
// The chip holds three of the small tiles' workgroups of four waves a CU, one or two of eight (their registers), two of
// the fp32 ones of large tiles (256 rows over 16384 entries 226 us with places for one, 191 for two) and one of the
// bf16 ones, whose tiles fill LDS: with twice the places 256 rows over 16384 took 54 us for 41 (weights in one part), waiting for a second round.
inline SharedPlan plan_of(const SharedDims& sd, bool few, int waves) {
  SharedPlan p;
  p.few = few;
  p.waves = waves;
  p.rows = few ? 16 : 16 * waves;
  p.tiles = most_tiles(sd, p.rows) * sd.G;
  const int64_t target = few ? (waves == 8 ? 256 : 768) : (sd.dtype == 1 ? 256 : 512);
  // what row tiles' last, unfilled chunks take: all of them where one workgroup more is a second round (64 rows over 8192 entries
  // 30.2 and 21.4 us, 256 over 4096 25.2 and 23.0), half of them elsewhere (fp32, 256 over 1024 32.0 and 27.7)
  const int64_t last = !few && sd.dtype == 1 ? p.tiles : p.tiles / 2, room = target - last > target / 4 ? target - last : target / 4;
  p.places = (int)((p.tiles + room + 7) & ~(int64_t)7);
  return p;
}
// `entries`: rows of the packed arrays, the only length that the host has.  The rows and entries of a (group, KV head) are
// taken as the mean.  (Arrays that hold the entries of all layers look as many times too long, and the call takes the large tiles where small ones
// are faster: of 32 layers, 16 sequences over 1024 entries a head 14.6 us and 11.7 with the layer's rows alone, 64 over 512 17.6 and 12.3.)
// The thresholds are fitted to measurements of 288 shapes, over which the choice takes 1.01 times the better kernel's time in the mean; products
// count 16 rows by 32 keys, and where fp32 takes eight waves they count once more by the row tiles, each of which has states to join.  Small tiles spread little work over the chip with fewer states and one launch, large ones go through keys
// and values fewer times.  us, heads of 128, small tiles with four waves, with eight, large tiles:
//   bf16, 8 KV heads, 16 rows each: over 128 entries 9.3, 8.2, 12.6; 1024 11.4, 11.8, 13.1; 4096 18.7, 16.9, 16.9; 16384 27.4, 25.5, 27.2
//   64 rows: over 256 10.0, 10.6, 13.7; 2048 15.3, 14.0, 15.5; 4096 20.6, 17.0, 17.5; 8192 27.6, 37, 22.3
//   256 rows: over 512 14.6, 12.5, 17.9; 1024 19.7, 16.8, 18.5; 2048 24.2, 24.1, 21.1; 8192 49, 54, 29.7
//   4 rows: over 24000 (eight, large) 32.2, 34.7; 65536 64, 68; 16 rows: over 32768 37.6, 37.8; 65536 56, 55; 131072 134, 93
//   fp32, 16 rows: over 2048 17.8, 19.7, 18.9; 8192 27, 30, 35; 32 rows: over 4096 21.3, 23.7, 25.5; 16384 78, 55, 68
//   128 rows: over 256 10.9, 12.8, 16.1; 1024 21.1, 18.0, 22.6; 2048 28.8, 23.4, 26.0; 8192 71, 66, 58
// and heads of 64 (four waves; eight are slower at all sizes), 2 KV heads: 128 rows over 8192 15.8 and 17.0, 32 over 16384 18.7 and 16.4.
// Large tiles have 64 rows (four waves), in bf16 for more rows 128 (eight).
inline SharedPlan shared_plan(const SharedDims& sd, int64_t entries) {
  const bool bf = sd.dtype == 1;               // GRACEKV_BF16
  const bool wide = sd.d > 64;
  const int64_t heads = (int64_t)sd.n_group * sd.G, mean = ((int64_t)sd.n_seq * sd.hpg + sd.n_group - 1) / sd.n_group;
  const int64_t each = entries / heads, tiles = (mean + 15) / 16;
  const int64_t steps = tiles * ((entries < (int64_t)1 << 40 ? entries : (int64_t)1 << 40) / 32);       // products of 16 rows and 32 keys
  const bool little = steps <= (bf && !wide ? 10240 : 4352) && each <= (bf && wide ? 5120 : 10240);
  if (little || (bf ? mean <= 16 && each <= 32768 : mean <= 32)) {
    const bool eight = wide && (bf ? each > 1536 || each <= 160 || steps >= 960 : mean > 16 && steps * tiles * heads >= 35000);
    return plan_of(sd, true, eight ? 8 : 4);
  }
  return plan_of(sd, false, bf && mean > 64 ? 8 : 4);
}

}  // namespace gkv
