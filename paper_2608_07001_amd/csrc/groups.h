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
// mean.  Up to 16 rows are few, and up to 64 where they have few entries, which the small tiles spread
// over the chip with fewer states: the 8B heads, few and many, us: 1 sequence over 512 entries a head 8.8 and
// 13.9, 8 over 512 10.4 and 13.2, 16 over 2048 15.5 and 15.5, 16 over 16384 40 and 27; fp32 with 64 rows over 2000 12.3 and
// 15.2.  Beyond, four waves take 64 rows (bf16), eight 128.  The chip holds three of the
// few's workgroups a CU and one of the others (their tiles fill LDS): with twice the places 64 sequences over 16384
// entries took 54 us for 41, waiting for a second round.
inline SharedPlan shared_plan(const SharedDims& sd, int64_t entries) {
  const bool bf = sd.dtype == 1;               // GRACEKV_BF16
  const int64_t mean = ((int64_t)sd.n_seq * sd.hpg + sd.n_group - 1) / sd.n_group;
  SharedPlan p;
  p.few = mean <= 16 || (mean <= 64 && entries / ((int64_t)sd.n_group * sd.G) <= 2048);
  p.waves = !p.few && bf && mean > 64 ? 8 : 4;
  p.rows = p.few ? 16 : 16 * p.waves;
  p.tiles = most_tiles(sd, p.rows) * sd.G;
  const int64_t target = p.few ? 768 : 256;
  const int64_t room = target - p.tiles / 2 > target / 4 ? target - p.tiles / 2 : target / 4;
  p.places = (int)((p.tiles + room + 7) & ~(int64_t)7);
  return p;
}

}  // namespace gkv
