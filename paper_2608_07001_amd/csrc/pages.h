// Where a token lies in a paged cache, and which sequence a packed row belongs to:
// the index arithmetic of the append and paged attention kernels, plain C++ so that
// the host can run it as well.  Nothing here reads memory except through `cu`.
//
// A cache holds n_pages pages of `1 << shift` tokens, page_stride elements apart,
// each [G][1 << shift][d].  A sequence's row of the block table names its pages in
// order; a place whose id lies outside [0, n_pages) holds no page.
#pragma once

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

}  // namespace gkv
