// Internal interface between the host side of the paged cache (ff_paged.cpp) and its
// kernels.  Not part of the C ABI.
#pragma once

#include <float.h>
#include <math.h>

#include "ff_internal.h"
#include "ff_numeric.h"
#include "ff_paged.h"
#include "paged_plan.h"

namespace ff {

// Tensors of one attention launch.  q rows are q_stride elements apart; out is dense.
struct PagedTensors {
  const void* q;
  void* out;
  float* lse;               // optional [n_tokens][query heads]
  const void* k_pages;      // [num_pages][kv_heads][page tokens][d]
  const void* v_pages;
  float* part;              // partial results of items of tiles with several parts
  int64_t q_stride;
  float scale;              // softmax_scale
  float scale_log2;         // softmax_scale * log2 e
};

// Tensors of one append launch; rows are *_stride elements apart, q_out is dense.
struct PagedAppend {
  const void* q;            // optional
  const void* k;
  const void* v;
  void* q_out;
  void* k_pages;
  void* v_pages;
  const int32_t* positions; // optional [n_tokens][3]
  int64_t q_stride, k_stride, v_stride;
  int32_t n_t, n_th;        // pairs [0, n_t) turn by t, [n_t, n_th) by h, the rest by w
  double omega[64];         // frequency of each pair
};

// lds_copy_blocks (attn_tile.h) past the caches (NT): for keys that no other workgroup reads
template <int N, bool NT>
__device__ inline void paged_copy(uint32_t dst, const char* base, const uint32_t (&off)[N]) {
  static_assert(N == 2 || N == 4, "1 KB copies of 16 rows");
  if constexpr (!NT)
    lds_copy_blocks<N>(dst, base, off);
  else if constexpr (N == 2)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %1, %3 nt\n\t"
                 "global_load_lds_dwordx4 %2, %3 offset:1024 nt"
                 :: "s"(dst), "v"(off[0]), "v"(off[1]), "s"(base) : "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\t"
                 "global_load_lds_dwordx4 %1, %5 nt\n\t"
                 "global_load_lds_dwordx4 %2, %5 offset:%6 nt\n\t"
                 "global_load_lds_dwordx4 %3, %5 offset:%7 nt\n\t"
                 "global_load_lds_dwordx4 %4, %5 offset:%8 nt"
                 :: "s"(dst), "v"(off[0]), "v"(off[1]), "v"(off[2]), "v"(off[3]), "s"(base),
                    "n"(1 * 1024), "n"(2 * 1024), "n"(3 * 1024) : "memory");
}

constexpr int kPagedPromptRows = 256;   // rows of a tile of launch_paged_prompt

// Two bf16 in a word: whether one is not finite, and the word with those zeroed
__device__ inline bool bf16_pair_not_finite(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ inline uint32_t bf16_pair_finite(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
  return w;
}

// Floats of one partial result: the output [rt][d] of its keys alone, then the reference and the
// sum of the weights of each row.  Parts are joined as the convex combination of their outputs, as
// are the waves of a workgroup: sums of weighted values that are not yet divided would pass
// float32's range where values are near its end.
__host__ __device__ inline int64_t paged_part_floats(int rt, int d) { return int64_t(rt) * (d + 2); }

// 1 / l, 0 for the sum of a row that saw nothing
__device__ inline float paged_inverse(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// N elements of a row of the output
template <class T, int N>
__device__ inline void paged_store(T* out, const float* v) {
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const u32x2 w = {pack_bf16_rne(v[i], v[i + 1]), pack_bf16_rne(v[i + 2], v[i + 3])};
      *reinterpret_cast<u32x2*>(out + i) = w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4)
      *reinterpret_cast<f32x4*>(out + i) = f32x4{v[i], v[i + 1], v[i + 2], v[i + 3]};
  }
}

// base-2 log-sum-exp of a row from its reference and sum (-inf for a row that saw nothing)
__device__ inline float paged_lse(float m, float u) { return u == 0.0f ? -INFINITY : m + log2f(u); }

hipError_t launch_paged_append(const PagedBatch& b, const PagedAppend& a, int head_dim, int dtype,
                               hipStream_t stream);

// Few rows per sequence: tiles of 16 qt rows, keys split as sp says; items: the launch's
// items per kv head (paged_max_items); waves: 2 or 4 per workgroup; once: no key is read by
// two tiles.
hipError_t launch_paged_attn_bf16(int qt, int waves, bool once, const PagedBatch& b,
                                  const PagedSplit& sp, const PagedTensors& t, int64_t items, int head_dim,
                                  hipStream_t stream);
hipError_t launch_paged_attn_f32(int qt, bool once, const PagedBatch& b, const PagedSplit& sp,
                                 const PagedTensors& t, int64_t items, int head_dim,
                                 hipStream_t stream);

// Many rows per sequence (bf16): tiles of kPagedPromptRows rows.
hipError_t launch_paged_prompt(const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                               int64_t items, int head_dim, hipStream_t stream);

// Joins the parts that those launches left: tiles of `rows` rows, about `used` of them
// used, at most `tiles` tiles per kv head.
hipError_t launch_paged_join(int rows, int used, const PagedBatch& b, const PagedSplit& sp,
                             const PagedTensors& t, int64_t items, int64_t tiles, int head_dim,
                             int dtype, hipStream_t stream);

}  // namespace ff
