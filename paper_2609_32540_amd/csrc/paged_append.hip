// Appending new tokens to a paged cache: K is rotated by the token's position and written
// with V to the token's place in its sequence's pages; Q, when given, is rotated into a
// dense array of its own.
//
// The rotation is ff_rope3d's (ff_numeric.h: float64, rounded once), its angles computed
// once per (token, pair) in float64 and kept in LDS for every head.  Bound by HBM: each
// row is read once and written once, in 16-byte vectors.  One block of 256 threads takes
// a few consecutive rows of the batch.  Which sequence a row belongs to is not passed:
// every wave counts the sequences that end at or before it (q_start read one element per
// lane, a ballot per row), so that a captured graph follows the device's lengths.

#include <hip/hip_runtime.h>

#include "ff_paged_internal.h"

namespace ff {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kMaxTok = 8;    // rows of the batch per block

template <class T, int D>
__global__ __launch_bounds__(kThreads)
void paged_append_kernel(PagedBatch b, PagedAppend a, int tok_per_block) {
  constexpr int P = D / 2;
  constexpr int EPV = 16 / sizeof(T);   // elements per 16-byte vector
  constexpr int VPR = D / EPV;          // vectors per head row
  __shared__ double2 cs_d[kMaxTok][P];
  __shared__ int64_t dst[kMaxTok];      // element offset of kv head 0's row in the pools, -1: none
  __shared__ int32_t idx[kMaxTok];      // index of the token in its sequence, -1: no such token
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = blockIdx.x * tok_per_block;
  const int n_rows = min(tok_per_block, b.n_tokens - row0);
  const int page_tokens = 1 << b.page_shift;

  for (int r = wave; r < n_rows; r += kWaves) {
    const int row = row0 + r;
    int s = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
      const bool ended = s0 + lane < b.n_seqs && b.q_start[s0 + lane + 1] <= row;
      s += __builtin_popcountll(__builtin_amdgcn_ballot_w64(ended));
    }
    int index = -1;
    int64_t at = -1;
    if (s < b.n_seqs) {
      const PagedSeq q = paged_seq(b, s);
      if (row >= q.q0 && row < q.q0 + q.n_new) index = q.first + (row - q.q0);
      if (index >= 0) {
        const int page = paged_page(b, s, index);
        if (page >= 0)
          at = (int64_t(page) * b.kv_heads * page_tokens + (index & (page_tokens - 1))) * D;
      } else {
        index = -1;
      }
    }
    if (lane == 0) {
      idx[r] = index;
      dst[r] = at;
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n_rows * P; e += kThreads) {
    const int r = e / P, pair = e % P;
    int pos = idx[r];
    if (pos >= 0 && a.positions != nullptr)
      pos = a.positions[int64_t(row0 + r) * 3 + (pair < a.n_t ? 0 : (pair < a.n_th ? 1 : 2))];
    double s, c;
    sincos(double(pos) * a.omega[pair], &s, &c);
    cs_d[r][pair] = make_double2(c, s);
  }
  __syncthreads();
  const int q_heads = a.q != nullptr ? b.kv_heads * b.group : 0;
  const int vecs = (q_heads + 2 * b.kv_heads) * VPR;   // of one row of the batch
  for (int i = threadIdx.x; i < n_rows * vecs; i += kThreads) {
    const int r = i / vecs, v = i - r * vecs;
    if (idx[r] < 0) continue;
    const int64_t row = row0 + r;
    const int c = v % VPR;
    int h = v / VPR;
    if (h < q_heads) {
      const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.q) + row * a.q_stride + h * D + c * EPV);
      *reinterpret_cast<uint4*>(static_cast<T*>(a.q_out) + (row * q_heads + h) * D + c * EPV) =
          rotate_vec<T>(x, cs_d[r] + c * (EPV / 2));
      continue;
    }
    if (dst[r] < 0) continue;
    h -= q_heads;
    const bool is_v = h >= b.kv_heads;
    if (is_v) h -= b.kv_heads;
    const int64_t at = dst[r] + int64_t(h) * page_tokens * D + c * EPV;
    if (is_v) {
      *reinterpret_cast<uint4*>(static_cast<T*>(a.v_pages) + at) =
          *reinterpret_cast<const uint4*>(static_cast<const T*>(a.v) + row * a.v_stride + h * D + c * EPV);
    } else {
      const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const T*>(a.k) + row * a.k_stride + h * D + c * EPV);
      *reinterpret_cast<uint4*>(static_cast<T*>(a.k_pages) + at) = rotate_vec<T>(x, cs_d[r] + c * (EPV / 2));
    }
  }
}

}  // namespace

hipError_t launch_paged_append(const PagedBatch& b, const PagedAppend& a, int head_dim, int dtype,
                               hipStream_t stream) {
  const int per = 2;
  const dim3 grid(unsigned((b.n_tokens + per - 1) / per));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, b, a, per);
    return hipGetLastError();
  };
  if (dtype == FF_DT_BF16)
    return head_dim == 64 ? go(paged_append_kernel<__bf16, 64>) : go(paged_append_kernel<__bf16, 128>);
  return head_dim == 64 ? go(paged_append_kernel<float, 64>) : go(paged_append_kernel<float, 128>);
}

}  // namespace ff
