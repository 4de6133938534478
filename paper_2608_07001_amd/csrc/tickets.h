// How workgroups that each leave a state in a workspace find the one that comes last, which
// joins them, without a second launch.
#pragma once

#include "serve.h"

namespace gkv {

static inline size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }

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
// RAISED: raise() came before, by the same thread
__device__ __forceinline__ void raise(unsigned long long* word) {
  __hip_atomic_fetch_max(word, PA_BASE, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
template <bool RAISED> __device__ __forceinline__ bool last_of(unsigned long long* word, int parts) {
  const unsigned long long end = PA_BASE + parts - 1;
  unsigned long long was;
  if (!RAISED) raise(word);
  for (;;) {
    was = __builtin_amdgcn_atomic_inc64((unsigned long*)word, end, __ATOMIC_RELAXED, "agent");
    if (was <= end && was >= PA_BASE) return was == end;
    raise(word);                              // below: put to 0 by another between the two steps
  }
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

}  // namespace gkv
