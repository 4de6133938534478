// Declarations shared by the operators around the compressed cache: attention over
// prompts (prompt.hip), appending to pages (append.hip) and attention over pages
// (paged.hip).
#pragma once

#include <type_traits>

#include "common.h"
#include "pages.h"

namespace gkv {

// strides in elements
struct AppendDims {
  int64_t n_new, rope_rows;
  int64_t k_tok, k_head, v_tok, v_head, q_tok, q_head, o_tok, o_head;
};
struct PromptDims {
  int dtype, G, H, d, hpg, n_seq;
  int64_t n_q, n_k;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;
};
constexpr int64_t PR_STRIDE = 1 << 24;    // longest distance of two rows of a prompt's keys or values
// the packed entries in front of the pages (all null: none)
struct PrefixView {
  const int64_t* start;
  const int64_t* count;
  const void* K;
  const void* V;
  const float* logm;
  int64_t rows;
};

hipError_t launch_append(const PageDims& pg, const AppendDims& ap, const void* k, const void* v, const void* q,
                         const int32_t* table, const int32_t* start, const int32_t* cu, const int32_t* pos,
                         const float* cosT, const float* sinT, void* Kp, void* Vp, void* q_out, hipStream_t st);
size_t prompt_ws_bytes(const PromptDims& pd);
int64_t prompt_items(const PromptDims& pd);      // workgroups of its launch
hipError_t launch_prompt(const PromptDims& pd, const void* q, const void* k, const void* v, const int32_t* cu_q,
                         const int32_t* cu_k, void* out, float* lse, void* ws, hipStream_t st);
size_t paged_ws_bytes(const PageDims& pg);
int64_t paged_items(const PageDims& pg);         // at most so many workgroups
hipError_t launch_paged(const PageDims& pg, int64_t q_tok, const void* q, const void* Kp, const void* Vp,
                        const int32_t* table, const int32_t* len, const PrefixView& px, void* out, float* lse, void* ws,
                        hipStream_t st);

// two floats to bf16, nearest even, low half first
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 x = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
}

// the sequence b in [0, n) whose span could hold row t: the last with cu[b] <= t (0 if
// none has).  A wave asks 64 places at a time, so up to 64 sequences take one load.
// Every lane of the wave calls it with the same arguments.  The starts have to ascend: the
// places that hold are counted.  Otherwise it gives some b in [0, n), and its caller leaves
// out a row that is not in the span of that one.
template <typename F>
__device__ __forceinline__ int find_last(int n, F at_most) {   // at_most(b): start of b <= what is looked for; falling
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = n;                                          // the answer + 1 lies in [lo, hi]
  while (hi - lo > 0) {
    const int step = (hi - lo + 63) / 64;
    const int b = lo + lane * step;
    const uint64_t yes = __ballot(b < hi && at_most(b));
    const int k = __popcll(yes);                               // the first k probes hold
    if (k == 0) break;
    const int a = lo + (k - 1) * step + 1;                     // (k - 1)'s place holds
    hi = min(hi, lo + k * step);                               // k's place does not
    lo = a;
    if (step == 1) break;
  }
  return __builtin_amdgcn_readfirstlane(lo > 0 ? lo - 1 : 0);
}
// the same, each lane for a row of its own
__device__ __forceinline__ int span_with(const int32_t* cu, int n, int64_t t) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (cu[mid] <= t) lo = mid + 1; else hi = mid;
  }
  return lo > 0 ? lo - 1 : 0;
}
__device__ __forceinline__ int find_span(const int32_t* cu, int n, int64_t t) {
  return find_last(n, [&](int b) { return cu[b] <= t; });
}

}  // namespace gkv
