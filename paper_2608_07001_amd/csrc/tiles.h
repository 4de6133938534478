// Tiles of keys and values in LDS and their 32x32 matrix products, for the attention of
// prompts (prompt.hip) and over shared entries (shared.hip).
#pragma once

#include "serve.h"

namespace gkv {

typedef float f32x16 __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16 mfma_bf16_32x32x16(uint4 a, uint4 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// the stated wait for the matrix pipeline (mfma_done) for these accumulators
__device__ __forceinline__ void mfma_done16(f32x16& x) { asm volatile("s_nop 15\n\ts_nop 4" : "+v"(x)); }

// Orders a block's N products, M at a time on the same operand, and their LDS reads (R for each M): the reads AHEAD of them early.
template <int N, int R, int AHEAD, int M = 1> __device__ __forceinline__ void reads_ahead() {
  constexpr int A = AHEAD < N ? AHEAD : N;
  __builtin_amdgcn_sched_group_barrier(0x100, R * A, 0);        // LDS reads
#pragma unroll
  for (int i = 0; i < N - A; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, M, 0);          // products
    __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, M * A, 0);
}

// 16 bytes of a tile
__device__ __forceinline__ uint4 lds_at(const uint4* tile, int byte) { return *(const uint4*)((const char*)tile + byte); }
// the four 16-bit values of a lane after the transposing read: `byte` is where the lane's 8
// bytes of its group's 4 x 16 block lie (lanes 4 r .. 4 r + 3: row r), returned is column lane % 16
__device__ __forceinline__ uint2 lds_read_tr(const uint4* tile, int byte) {
  auto q = (__attribute__((address_space(3))) s16x4*)((const char*)tile + byte);
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(q));
}

// The rows of one key tile as a bounded buffer: `rows` rows of D elements, `tok` elements
// apart; a load past the last row gives 0.  (tok is at most PR_STRIDE, so the bytes of a
// tile fit 31 bits.)
typedef __amdgpu_buffer_rsrc_t Buffer;
template <typename T, int D>
__device__ __forceinline__ Buffer tile_buffer(const T* base, int64_t tok, int rows) {
  const int bytes = (int)(((int64_t)(rows - 1) * tok + D) * (int64_t)sizeof(T));
  return __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00020000);
}
// 16 bytes a lane straight into LDS, lane l to dst + l (dst: the same for the wave); the
// wave's vector memory counter says when they are there
__device__ __forceinline__ void buffer_load_lds(Buffer b, uint4* dst, int off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b, (__attribute__((address_space(3))) void*)dst, 16, off, 0, 0, 0);
}

// Workgroup barrier behind the wave's LDS accesses and its loads into LDS but for the last N vector
// memory operations.  (A fence, as __syncthreads() has it, would wait for those as well.)
template <int N> __device__ __forceinline__ void loaded_barrier() {
  static_assert(N >= 0 && N < 64, "the counter's range");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (N & 15) | (N >> 4) << 14);      // s_waitcnt vmcnt(N) lgkmcnt(0)
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// place of 16-byte piece c of key row t in a staged tile: neighbouring rows start in
// other banks, for the reads along a row (16 rows, one piece) and the transposing ones
// (8 rows, four pieces)
template <int D> __device__ __forceinline__ int swz(int t, int c) {
  if constexpr (D == 128) return t * 16 + (c ^ (((t & 3) << 2) | ((t >> 2) & 3)));
  else return t * 8 + (c ^ ((((t >> 1) & 1) << 2) | ((t >> 2) & 3)));
}

}  // namespace gkv
