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
// `entries`: rows of the packed arrays.  The rows and entries of a (group, KV head) are taken as the
// mean.  Small tiles spread little work over the chip with fewer states and one launch, large ones go through keys
// and values fewer times.  us, small and large tiles, bf16, heads of 128: 4 to 16 rows over 1024 entries 11 and 13, over
// 16384 25 to 27 and 24 to 26, over 65536 78 and 52 to 64; 64 rows of 8 KV heads over 1024 11.9 and 14.5, over 4096 20.8 and
// 17.2; 128 over 2048 17.1 and 18.2; 256 over 512 14.7 and 17.5, over 2048 24.7 and 20.6; heads of 64, 2 KV heads,
// 128 rows over 8192 15.8 and 16.5, 32 over 16384 18.6 and 16.0.  fp32, heads of 128: 8 rows over 65536 124 and 212, 64 over
// 1024 14.6 and 18.0, over 4096 30.1 and 27.9; 256 over 512 20.8 and 21.7, over 2048 46 and 42.
// Large tiles have 64 rows (four waves), in bf16 for more rows 128 (eight).  The chip holds three of the
// small ones' workgroups a CU, two of the fp32 ones (256 rows over 16384 entries 226 us with places for one, 191 for two,
// over 2048 43.8 and 42.3) and one of the others, whose tiles fill LDS: with twice the places 256 rows over 16384
// took 54 us for 41, waiting for a second round.
inline SharedPlan shared_plan(const SharedDims& sd, int64_t entries) {
  const bool bf = sd.dtype == 1;               // GRACEKV_BF16
  const int64_t mean = ((int64_t)sd.n_seq * sd.hpg + sd.n_group - 1) / sd.n_group;
  SharedPlan p;
  const int64_t each = entries / ((int64_t)sd.n_group * sd.G), tiles = (mean + 15) / 16, wide = sd.d / 64;
  // in products of 16 rows, 32 keys and 64 dims, and where no row has a long way to go
  const bool little = entries / 32 <= (bf ? 10240 : 5120) / (tiles * wide) && each <= (bf && wide > 1 ? 2560 : 10240);
  p.few = little || (bf ? mean <= 16 && each <= 32768 : mean <= 32);
  p.waves = !p.few && bf && mean > 64 ? 8 : 4;
  p.rows = p.few ? 16 : 16 * p.waves;
  p.tiles = most_tiles(sd, p.rows) * sd.G;
  const int64_t target = p.few ? 768 : (bf ? 256 : 512);
  const int64_t room = target - p.tiles / 2 > target / 4 ? target - p.tiles / 2 : target / 4;
  p.places = (int)((p.tiles + room + 7) & ~(int64_t)7);
  return p;
}

}  // namespace gkv
