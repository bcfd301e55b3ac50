// Appending new tokens to a paged cache: K is rotated by the token's position and written
// with V to the token's place in its sequence's pages; Q, when given, is rotated into a
// dense array of its own.
//
// The rotation is ff_rope3d's (ff_numeric.h: float64, rounded once), its angles computed
// once per (token, pair) in float64 and kept in LDS for every head.  Bound by HBM where
// there is much to move: each row is read once and written once, in 16-byte vectors.  One
// block of 256 threads takes a few consecutive rows of the batch.  Which sequence a row
// belongs to is not passed: a wave counts the sequences that end at or before it (q_start
// read one element per lane, a ballot per 64), so that a captured graph follows the
// device's lengths.  A small call is a chain of latencies (q_start, kv_len, the page table,
// the angles), so what does not hang on it, the first U vectors of every thread, is
// loaded ahead of it.

#include <hip/hip_runtime.h>

#include "ff_paged_internal.h"

namespace ff {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kUnroll = 4;    // vectors per thread in flight

// R: rows of the batch per block (rows_per_block)
template <class T, int D, int R>
__global__ __launch_bounds__(kThreads)
void paged_append_kernel(PagedBatch b, PagedAppend a) {
  constexpr int P = D / 2;
  constexpr int EPV = 16 / sizeof(T);   // elements per 16-byte vector
  constexpr int VPR = D / EPV;          // vectors per head row
  constexpr int U = kUnroll;
  __shared__ double2 cs_d[R][P];
  __shared__ int64_t dst[R];      // element offset of kv head 0's row in the pools, -1: none
  __shared__ int32_t idx[R];      // index of the token in its sequence, -1: no such token
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row0 = blockIdx.x * R;
  const int n_rows = min(R, b.n_tokens - row0);
  const int page_tokens = 1 << b.page_shift;
  const int q_heads = a.q != nullptr ? b.kv_heads * b.group : 0;
  const int vecs = (q_heads + 2 * b.kv_heads) * VPR;   // of one row: Q, then K, then V
  const int total = n_rows * vecs;

  auto row_of = [&](int i) __attribute__((always_inline)) {
    return R == 2 && i >= vecs ? 1 : 0;
  };
  auto load = [&](int i) __attribute__((always_inline)) {
    const int r = row_of(i), v = i - r * vecs, c = v % VPR;
    const int64_t row = row0 + r;
    const int h = v / VPR, hk = h - q_heads, hv = hk - b.kv_heads;
    const T* p = hk < 0 ? static_cast<const T*>(a.q) + row * a.q_stride + h * D
                 : hv < 0 ? static_cast<const T*>(a.k) + row * a.k_stride + hk * D
                          : static_cast<const T*>(a.v) + row * a.v_stride + hv * D;
    return *reinterpret_cast<const uint4*>(p + c * EPV);
  };
  uint4 x[U];
#pragma unroll
  for (int u = 0; u < U; ++u) x[u] = load(min(int(threadIdx.x) + u * kThreads, total - 1));

  for (int r = wave; r < n_rows; r += kWaves) {
    const int row = row0 + r;
    int s = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += 256) {
      int end[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) end[k] = b.q_start[min(s0 + 64 * k + lane, b.n_seqs - 1) + 1];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        s += __builtin_popcountll(__builtin_amdgcn_ballot_w64(s0 + 64 * k + lane < b.n_seqs && end[k] <= row));
    }
    int index = -1;
    int64_t at = -1;
    if (s < b.n_seqs) {
      const PagedSeq q = paged_seq(b, s);
      if (row >= q.q0 && row < q.q0 + q.n_new) index = max(q.first + (row - q.q0), -1);
      if (index >= 0) {
        const int page = paged_page(b, s, index);
        if (page >= 0)
          at = (int64_t(page) * b.kv_heads * page_tokens + (index & (page_tokens - 1))) * D;
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

  auto put = [&](int i, uint4 w) __attribute__((always_inline)) {
    const int r = row_of(i), v = i - r * vecs, c = v % VPR;
    if (idx[r] < 0) return;
    const int64_t row = row0 + r;
    const int h = v / VPR, hk = h - q_heads, hv = hk - b.kv_heads;
    if (hv < 0) w = rotate_vec<T>(w, cs_d[r] + c * (EPV / 2));
    T* p;
    if (hk < 0) {
      p = static_cast<T*>(a.q_out) + (row * q_heads + h) * D;
    } else {
      if (dst[r] < 0) return;
      p = hv < 0 ? static_cast<T*>(a.k_pages) + dst[r] + int64_t(hk) * page_tokens * D
                 : static_cast<T*>(a.v_pages) + dst[r] + int64_t(hv) * page_tokens * D;
    }
    // (past the caches: 9 and 20% less at 40 + 2 x 40 heads x 128, 4680 tokens and 20 + 2 x 5, 2300)
    __builtin_nontemporal_store(u32x4{w.x, w.y, w.z, w.w}, reinterpret_cast<u32x4*>(p + c * EPV));
  };
  for (int base = threadIdx.x; base < total; base += U * kThreads) {
    uint4 y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) y[u] = x[u];
    if (base + U * kThreads < total)   // the next ones, while these are rotated and stored
#pragma unroll
      for (int u = 0; u < U; ++u) x[u] = load(min(base + (U + u) * kThreads, total - 1));
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (base + u * kThreads < total) put(base + u * kThreads, y[u]);
  }
}

// Rows per block: 2 where that gives a thread no more than its kUnroll vectors and leaves a
// block per CU, else 1 (12 + 2 x 4 heads x 64, float32, 1000 rows 7.9 us with 1 and 6.7
// with 2; 9 + 2 x 3 heads x 128, 6400 rows 18.2 and 15.3; 32 + 2 x 8 heads x 128, 200 rows
// 6.2 and 8.2; four gain nothing: 16 + 2 x 8 heads x 64, 900 rows 6.3 with 2, 7.2 with 4).
int rows_per_block(int n_tokens, int vecs) {
  return 2 * vecs <= kUnroll * kThreads && n_tokens / 2 >= device_cus() ? 2 : 1;
}

template <class T, int D>
hipError_t launch(const PagedBatch& b, const PagedAppend& a, hipStream_t stream) {
  const int heads = (a.q != nullptr ? b.kv_heads * b.group : 0) + 2 * b.kv_heads;
  const int per = rows_per_block(b.n_tokens, heads * D * int(sizeof(T)) / 16);
  const dim3 grid(unsigned((b.n_tokens + per - 1) / per));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, b, a);
    return hipGetLastError();
  };
  return per == 2 ? go(paged_append_kernel<T, D, 2>) : go(paged_append_kernel<T, D, 1>);
}

}  // namespace

hipError_t launch_paged_append(const PagedBatch& b, const PagedAppend& a, int head_dim, int dtype,
                               hipStream_t stream) {
  if (dtype == FF_DT_BF16)
    return head_dim == 64 ? launch<__bf16, 64>(b, a, stream) : launch<__bf16, 128>(b, a, stream);
  return head_dim == 64 ? launch<float, 64>(b, a, stream) : launch<float, 128>(b, a, stream);
}

}  // namespace ff
