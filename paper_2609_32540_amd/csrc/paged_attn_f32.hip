// Float32 attention over a paged cache, on the float32 matrix instructions
// (v_mfma_f32_16x16x4_f32): tiles, items, parts and masked keys as in paged_attn.hip, the
// operands as in attn_f32.hip.
//
// A workgroup of four waves runs one item; its 16-key blocks are dealt round robin to
// the waves.  A block lies in one page (pages hold multiples of 16 tokens), K and V go
// straight from global memory to the registers that the products read: the four summands
// of a product are chosen to be consecutive in memory, so one 16-byte load per lane feeds
// four products of each query tile.  The reference is subtracted from a score before the factor
// log2 e is applied, which rounds a difference of at most 4 above it instead of the score.
//
// One new token each of 16 sequences of up to 2300 tokens, 12 heads x 128: 51 us with the
// join = 4.5 TB/s (bound by HBM; workgroups of eight waves, one per CU instead of two, 6 us more);
// one block of 2184 tokens over 8736 keys, 3 heads: 284 us = 103 TFLOP/s (the float32 matrix
// rate, 153 TFLOP/s in a large product; beside the products an item costs about 5 us, and nine
// rounds of items are needed for an even load; the softmax among the next block's products, in
// a pipelined turn, gains nothing, nor do tiles of the same keys on one XCD, whose L2 serves 95%).

#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>

#include "ff_paged_internal.h"

namespace ff {
namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kBK = 16;                   // keys per block
constexpr float kLog2e = 1.44269504f;
constexpr float kRaise = 4.0f;            // natural units a score may pass the reference by: every
                                          // row's running max would move some row's O in most blocks

template <int D, int QT, bool NT>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_attn_f32_kernel(PagedBatch b, PagedSplit sp, PagedTensors t) {
  constexpr int KT = D / 16;              // 16-byte vectors of a K (or Q) row per lane
  constexpr int VH = D / 64;              // 16-byte vectors of a V row per lane
  constexpr int kRows = 16 * QT;          // rows of the workgroup
  constexpr int kPitch = D + 4;           // padded row of the join buffer (floats)
  __shared__ __attribute__((aligned(16))) float part[kWaves * kRows * kPitch];
  __shared__ float part_m[kWaves * kRows], part_l[kWaves * kRows];

  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
  const int head = blockIdx.x % b.kv_heads;
  const int item = blockIdx.x / b.kv_heads;

  PagedItem it;
  if (!PagedScan<kRows, kBK>(b, sp, lane).find(item, false, &it)) return;
  const int n_rows = it.seq.n_new * b.group;
  const int row0 = it.tile * kRows;
  const int row1 = min(row0 + kRows, n_rows) - 1;   // last row of the tile
  const PagedRange head_r = paged_range(b, it.seq, paged_token(b, row0));
  const PagedRange tail_r = paged_range(b, it.seq, paged_token(b, row1));
  const PagedBlocks<kBK> blocks = paged_blocks<kBK>(b, head_r, tail_r);
  const int t0 = uniform(int(int64_t(it.part) * blocks.n / it.parts));
  const int t1 = uniform(int(int64_t(it.part + 1) * blocks.n / it.parts));
  const bool rows_differ = head_r.hi != tail_r.hi || head_r.lo != tail_r.lo;

  f32x4 qreg[QT][KT];
  PagedRange see[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int r = min(row0 + 16 * x + l16, row1);
    const int tau = paged_token(b, r);
    see[x] = paged_range(b, it.seq, tau);
    const float* qp = static_cast<const float*>(t.q) + int64_t(it.seq.q0 + tau) * t.q_stride +
                      int64_t(head * b.group + r - tau * b.group) * D + 4 * grp;
#pragma unroll
    for (int i = 0; i < KT; ++i) qreg[x][i] = *reinterpret_cast<const f32x4*>(qp + 16 * i) * t.scale;
  }
  f32x4 o[QT][VH][4];
  float m_run[QT], l_run[QT];

  // lane i holds the page of block i of this wave's current 64 (a reload every 64 blocks)
  int page_of = -1;
  auto load_pages = [&](int i0) __attribute__((always_inline)) {
    const int tb = t0 + wave + kWaves * (i0 + lane);
    page_of = -1;
    if (tb < t1) page_of = paged_page(b, it.s, blocks.key0(tb));
  };
  const int slot_mask = (1 << b.page_shift) - 1;
  // elements from the pool's start to the 16 keys from key j, which lie in page `page`
  // (page 0 for a hole: masked)
  auto block_offset = [&](int page, int j) __attribute__((always_inline)) {
    return ((int64_t(max(page, 0)) * b.kv_heads + head) * (slot_mask + 1) + (j & slot_mask)) * D;
  };
  const float* kpool = static_cast<const float*>(t.k_pages);
  const float* vpool = static_cast<const float*>(t.v_pages);
  // 16 bytes per lane from a scalar base (the compiler would make vector addresses of the pool's
  // start and add to those); past the caches where no other workgroup reads the key
  using Base = const __attribute__((address_space(1))) char*;
  auto base_of = [](const float* p) __attribute__((always_inline)) {
    Base base = (Base)p;
    asm volatile("" : "+s"(base));
    return base;
  };
  auto load = [](Base base, uint32_t bytes) __attribute__((always_inline)) {
    const auto* v = (const __attribute__((address_space(1))) f32x4*)(base + bytes);
    return NT ? __builtin_nontemporal_load(v) : *v;
  };
  f32x4 kreg[KT], vreg[4][VH];
  const uint32_t k_lane = 4 * (l16 * D + 4 * grp), v_lane = 4 * (4 * grp * D + 4 * l16);   // bytes from a scalar base
  auto load_k = [&](int64_t off) __attribute__((always_inline)) {
    const Base p = base_of(kpool + off);
#pragma unroll
    for (int i = 0; i < KT; ++i) kreg[i] = load(p + 64 * i, k_lane);
  };
  auto load_v = [&](int64_t off) __attribute__((always_inline)) {
    const Base p = base_of(vpool + off);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int h = 0; h < VH; ++h) vreg[j][h] = load(p + 4 * (j * D + 64 * h), v_lane);
  };

  // The wave's blocks.  A wave whose O is not finite goes over them again, with a reference so
  // far above the scores that its weights sum to at most 1: O then stays below the largest
  // |V|, and is not finite where a V element is not.
  for (bool again = false;; again = true) {
    const float raise = again ? 0.0f : kRaise;
    const float lift = again ? (32 - __builtin_clz(uint32_t(kBK * (t1 - t0) | 1))) / kLog2e : 0.0f;
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      m_run[x] = -FLT_MAX;   // (finite: a key whose score is -inf then gets weight 0)
      l_run[x] = 0.0f;
#pragma unroll
      for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[x][h][e] = f32x4{};
    }
    int tb = t0 + wave, i = 0;
    int page = -1;
    int64_t off = 0;
    if (tb < t1) {
      load_pages(0);
      page = __builtin_amdgcn_readlane(page_of, 0);
      off = uniform(block_offset(page, blocks.key0(tb)));
      load_k(off);
      // (V behind K: the loop waits for K with V's loads in flight)
      __builtin_amdgcn_sched_barrier(0);
      load_v(off);
    }
    // Every turn issues the same loads in the same order, K of the next block, then its V (behind
    // the last one of page 0): so the waits for K leave V's loads in flight and the other way round.
    while (tb < t1) {
      f32x4 s[QT];
#pragma unroll
      for (int x = 0; x < QT; ++x) s[x] = f32x4{};
#pragma unroll
      for (int k = 0; k < KT; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int x = 0; x < QT; ++x)
            s[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(kreg[k][e], qreg[x][k][e], s[x], 0, 0, 0);
      const int j0 = blocks.key0(tb), cur = page;
      const int64_t cur_off = off;
      // the next block: its K now, its V once this block's V is consumed
      tb += kWaves;
      ++i;
      off = 0;
      if (tb < t1) {
        if ((i & 63) == 0) load_pages(i);
        page = __builtin_amdgcn_readlane(page_of, i & 63);
        off = uniform(block_offset(page, blocks.key0(tb)));
      }
      load_k(off);
      __builtin_amdgcn_sched_barrier(0);

      const bool edge = j0 + kBK > head_r.hi || cur < 0 || (j0 < tail_r.lo && j0 + kBK > b.anchor_tokens);
      bool spread = false;
      if (edge) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = j0 + 4 * grp + e;
#pragma unroll
          for (int x = 0; x < QT; ++x) {
            const bool seen = cur >= 0 && j < see[x].hi && (j >= see[x].lo || j < b.anchor_tokens);
            s[x][e] = seen ? s[x][e] : -INFINITY;
          }
          const bool any = cur >= 0 && j < tail_r.hi && (j >= head_r.lo || j < b.anchor_tokens);
          if (!any)
#pragma unroll
            for (int h = 0; h < VH; ++h) vreg[e][h] = f32x4{};
        }
        if (rows_differ) {
          bool bad = false;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int h = 0; h < VH; ++h)
#pragma unroll
              for (int w = 0; w < 4; ++w) bad |= !isfinite(vreg[e][h][w]);
          spread = __builtin_amdgcn_ballot_w64(bad) != 0;
          if (spread)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int h = 0; h < VH; ++h)
#pragma unroll
                for (int w = 0; w < 4; ++w) vreg[e][h][w] = isfinite(vreg[e][h][w]) ? vreg[e][h][w] : 0.0f;
        }
      }

      bool raised = false;
      float mx[QT];
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        mx[x] = max_across_groups(fmaxf(fmaxf(s[x][0], s[x][1]), fmaxf(s[x][2], s[x][3]))) + lift;
        raised |= mx[x] > m_run[x] + raise;   // (-FLT_MAX + raise is -FLT_MAX)
      }
      if (__builtin_amdgcn_ballot_w64(raised) != 0) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float m_new = mx[x] > m_run[x] + raise ? mx[x] : m_run[x];
          const float alpha = __builtin_amdgcn_exp2f((m_run[x] - m_new) * kLog2e);
          m_run[x] = m_new;
          l_run[x] *= alpha;
#pragma unroll
          for (int h = 0; h < VH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[x][h][e] *= alpha;
        }
      }
#pragma unroll
      for (int x = 0; x < QT; ++x) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          s[x][e] = __builtin_amdgcn_exp2f((s[x][e] - m_run[x]) * kLog2e);
        l_run[x] += (s[x][0] + s[x][1]) + (s[x][2] + s[x][3]);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int h = 0; h < VH; ++h)
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int x = 0; x < QT; ++x)
              o[x][h][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vreg[j][h][e], s[x][j], o[x][h][e], 0, 0, 0);
      if (spread) {
        // V elements that are not finite, for the rows that see their key
#pragma unroll 1
        for (int kk = 0; kk < kBK; ++kk) {
          const int j = j0 + kk;
          if (cur < 0 || j >= tail_r.hi) continue;
          const float* vr = vpool + cur_off + kk * D;
#pragma unroll
          for (int x = 0; x < QT; ++x) {
            float pr = 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) pr = e == (kk & 3) ? s[x][e] : pr;
            const float p = __shfl(pr, l16 + 16 * (kk >> 2));
            const bool seen = j < see[x].hi && (j >= see[x].lo || j < b.anchor_tokens);
#pragma unroll
            for (int h = 0; h < VH; ++h)
#pragma unroll
              for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const float v = vr[64 * h + 16 * grp + 4 * k + e];
                  if (seen && !isfinite(v)) o[x][h][e][k] += p * v;
                }
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
      load_v(off);
      __builtin_amdgcn_sched_barrier(0);
    }
    float any = 0.0f;
#pragma unroll
    for (int x = 0; x < QT; ++x)
#pragma unroll
      for (int h = 0; h < VH; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j) any = fmaf(o[x][h][e][j], 0.0f, any);
    if (again || __builtin_amdgcn_ballot_w64(any != 0.0f) == 0) break;
  }

  // join the waves
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const float l = sum_across_groups(l_run[x]);
    const int row = wave * kRows + 16 * x + l16;
    if (grp == 0) {
      part_m[row] = m_run[x];
      part_l[row] = l;
    }
#pragma unroll
    for (int h = 0; h < VH; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 w = {o[x][h][0][j], o[x][h][1][j], o[x][h][2][j], o[x][h][3][j]};
        *reinterpret_cast<f32x4*>(part + row * kPitch + 64 * h + 16 * grp + 4 * j) = w;
      }
  }
  __syncthreads();
  float* ws = t.part + (int64_t(item) * b.kv_heads + head) * paged_part_floats(kRows, D);
  for (int n = threadIdx.x; n < kRows * (D / 4); n += kThreads) {
    const int r = n / (D / 4), c = n % (D / 4);
    if (row0 + r > row1) continue;
    float m = part_m[r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part_m[w * kRows + r]);
    float l = 0.0f, a[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      a[w] = __builtin_amdgcn_exp2f((part_m[w * kRows + r] - m) * kLog2e);
      l += a[w] * part_l[w * kRows + r];
    }
    const float inv = paged_inverse(l);
    f32x4 acc = {};
    if (l != 0.0f)   // (a row that saw nothing is zero)
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
        acc += (a[w] * inv) * *reinterpret_cast<const f32x4*>(part + (w * kRows + r) * kPitch + 4 * c);
    if (it.parts > 1) {
      *reinterpret_cast<f32x4*>(ws + r * D + 4 * c) = acc;
      if (c == 0) {
        ws[kRows * D + r] = m;
        ws[kRows * D + kRows + r] = l;
      }
    } else {
      const int tau = paged_token(b, row0 + r);
      const int64_t at = int64_t(it.seq.q0 + tau) * (b.kv_heads * b.group) + head * b.group +
                         (row0 + r - tau * b.group);
      paged_store<float, 4>(static_cast<float*>(t.out) + at * D + 4 * c, reinterpret_cast<const float*>(&acc));
      if (t.lse != nullptr && c == 0) t.lse[at] = paged_lse(m * kLog2e, l);
    }
  }
}

// (tiles of 16 rows are chosen only where a sequence is one tile: once)
template <int D, int QT>
hipError_t launch(bool once, const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                  int64_t items, hipStream_t stream) {
  const dim3 grid(unsigned(items * b.kv_heads));
  if (QT == 1 || once)
    hipLaunchKernelGGL((paged_attn_f32_kernel<D, QT, true>), grid, dim3(kThreads), 0, stream, b, sp, t);
  else if constexpr (QT > 1)
    hipLaunchKernelGGL((paged_attn_f32_kernel<D, QT, false>), grid, dim3(kThreads), 0, stream, b, sp, t);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn_f32(int qt, bool once, const PagedBatch& b, const PagedSplit& sp,
                                 const PagedTensors& t, int64_t items, int head_dim,
                                 hipStream_t stream) {
  if (head_dim == 64) return qt == 2 ? launch<64, 2>(once, b, sp, t, items, stream) : launch<64, 1>(once, b, sp, t, items, stream);
  return qt == 2 ? launch<128, 2>(once, b, sp, t, items, stream) : launch<128, 1>(once, b, sp, t, items, stream);
}

}  // namespace ff
