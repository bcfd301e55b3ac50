// Attention of one or a few new tokens per sequence over a paged cache, bf16: the cache's
// length is split over workgroups and over the waves of a workgroup, and joined.
//
// Mathematics.  out = sum_j p_j v_j / sum_j p_j with p_j = 2^(c q.k_j - m), c = scale
// log2 e.  Any split of the keys works with a reference m of its own: waves, and parts, join as
// out = sum_w (2^(m_w - M) l_w / l) out_w, l = sum_w 2^(m_w - M) l_w, M = max m_w.
//
// Work split.  The query heads of one kv head read the same keys, so a tile is 16 QT rows
// (token, query head of the group) of one sequence and kv head.  An item is a tile and one
// of its parts of the keys (paged_plan.h); a workgroup of four waves runs one item of one
// kv head, 32-key blocks dealt round robin to its waves, which join through LDS; items of
// a tile with several parts leave float32 partial results in the workspace, joined
// by paged_join_kernel.  What bounds it: every key and value is read from HBM once, while
// the products fill the matrix unit's 16 columns with as few as one row.
//
// Operands as in attn_bf16_split.hip: S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_16x16x32_bf16; each wave copies its own blocks HBM -> LDS in whole pieces of
// rows (global_load_lds) and takes them into registers before the products, which frees
// the LDS for the copy of its next block.  A page holds the rows of one kv head in one
// piece ([kv heads][page tokens][d]), and at least 16 of them, so that each half of a
// block (16 keys) lies in one page and is copied from one base; rows of the page behind
// the sequence's end are copied with it and masked.
//
// Masked keys.  A key that no row of the tile sees (behind the end, in a hole, outside
// window and anchors) has its score replaced by -inf and its V row by zero: what its
// memory holds (stale values, infinities, NaN) does not matter.  Where the rows of a tile
// see different keys, a V element that is not finite is kept out of the products, which
// would spread it to every row as 0 * inf, and added for the rows that see it.
//
// Rounding: a probability enters the matrix unit as two bf16, its value rounded and what
// that leaves rounded again (2^-17 in all), since products cost nothing here: the output has
// the error of its own rounding, 1.7e-3 (relative-L2) where probabilities of one bf16 give
// 2.3e-3.  Scores, references, sums and O are float32.
//
// Range: an element of O is below the sum of weight times |V|, which a second run with weights
// that sum to at most 1 keeps finite, and joins add outputs, not sums: |V| up to 2^127 gives
// finite results.
//
// Measured (32/8 heads x 128, passes among others, joins included).  64 sequences of 150 to
// 12000 tokens: 244 us = 6.2 TB/s, 242 the copies alone (the kernel without its operand reads and
// products); read through the caches 274 us, so a key that no other tile reads is read past
// them.  One sequence of 32774 tokens: 31 us, of which the join is 5 to 6 (1.3 its launch, 0.7
// the lookup), 29 with the copies alone; 34 through the caches; 36 with twice the parts.  Two
// waves per workgroup, four workgroups per CU: 258 and 31, but 45 instead of 63 for 250 sequences
// of up to 308 tokens, 12 kv heads (and so they are chosen there).

#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>

#include <type_traits>

#include "ff_paged_internal.h"

namespace ff {
namespace {

constexpr int kBK = 32;            // keys per block
constexpr float kRaise = 56.0f;    // log2 units a score may exceed the reference by: sums of
                                   // 2^56 times the keys stay far inside float32

template <int D, int QT, int kWaves>
struct PagedCfg {
  static constexpr int KS = D / 32;            // 32-wide d slices of S^T
  static constexpr int DT = D / 16;            // 16-row d tiles of O^T
  static constexpr int BLOCK = kBK * 2 * D;    // bytes of one K (or V) block
  static constexpr int HALF = BLOCK / 2;       // of its half, 16 keys
  static constexpr int N = HALF / 1024;        // 1 KB copies of a half
  static constexpr int kRows = 16 * QT;
  static constexpr int kPitch = D + 4;         // padded row of the join buffer (floats)
  static constexpr int kJoin = kWaves * kRows * (kPitch + 2) * 4;
  static constexpr int kLds = kWaves * 2 * BLOCK > kJoin ? kWaves * 2 * BLOCK : kJoin;
};

template <int D, int QT, int kWaves, bool NT>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_attn_kernel(PagedBatch b, PagedSplit sp, PagedTensors t) {
  using C = PagedCfg<D, QT, kWaves>;
  constexpr int kThreads = 64 * kWaves;
  __shared__ __attribute__((aligned(1024))) char lds[C::kLds];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
  const int head = blockIdx.x % b.kv_heads;
  const int item = blockIdx.x / b.kv_heads;

  PagedItem it;
  if (!PagedScan<C::kRows, kBK>(b, sp, lane).find(item, false, &it)) return;
  const int n_rows = it.seq.n_new * b.group;
  const int row0 = it.tile * C::kRows;
  const int row1 = min(row0 + C::kRows, n_rows) - 1;   // last row of the tile
  const PagedRange head_r = paged_range(b, it.seq, paged_token(b, row0));
  const PagedRange tail_r = paged_range(b, it.seq, paged_token(b, row1));
  const PagedBlocks<kBK> blocks = paged_blocks<kBK>(b, head_r, tail_r);
  const int t0 = uniform(int(int64_t(it.part) * blocks.n / it.parts));
  const int t1 = uniform(int(int64_t(it.part + 1) * blocks.n / it.parts));
  const bool rows_differ = head_r.hi != tail_r.hi || head_r.lo != tail_r.lo;

  // Q^T operand and what each row sees (lane l16 of query tile x: row 16 x + l16)
  bf16x8 qreg[QT][C::KS];
  PagedRange see[QT];
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int r = min(row0 + 16 * x + l16, row1);
    const int tau = paged_token(b, r);
    see[x] = paged_range(b, it.seq, tau);
    const __bf16* qp = static_cast<const __bf16*>(t.q) + int64_t(it.seq.q0 + tau) * t.q_stride +
                       int64_t(head * b.group + r - tau * b.group) * D + 8 * grp;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) qreg[x][s] = *reinterpret_cast<const bf16x8*>(qp + 32 * s);
  }

  f32x4 o[C::DT][QT];
  float m_run[QT], l_run[QT];

  // Pages of this wave's blocks t0 + wave, + 4, ..: lane 2 i + half holds the page of that
  // half of block i of the current 32 (a reload every 32 blocks)
  int page_of = -1;
  auto load_pages = [&](int i0) __attribute__((always_inline)) {
    const int tb = t0 + wave + kWaves * (i0 + (lane >> 1));
    page_of = -1;
    if (tb < t1) {
      const int j = blocks.key0(tb) + 16 * (lane & 1);
      if (j < tail_r.hi) page_of = paged_page(b, it.s, j);
    }
  };

  // The wave's K and V block in LDS, in the layouts of attn_bf16_split.hip (lanes of a
  // quad (K) or octet (V) take consecutive bytes of a row, permuted so that the operand
  // reads are free of bank conflicts).
  char* kbuf = lds + wave * 2 * C::BLOCK;
  char* vbuf = kbuf + C::BLOCK;
  const int k_lane = 64 * l16 + 16 * (grp ^ (l16 >> 2));
  int v_lane[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int r = 4 * grp + (l16 >> 2);
    v_lane[p] = (r >> 3) * (16 * D) + 128 * (r & 7) + 32 * (p ^ ((r & 7) >> 1)) + 8 * (l16 & 3);
  }
  uint32_t koff[C::N], voff[C::N];
#pragma unroll
  for (int i = 0; i < C::N; ++i) {
    constexpr uint32_t kSpan = 1024u * (C::N - 1);
    const int kr = lane >> 2, kch = 4 * i + ((lane & 3) ^ (lane >> 4));
    const int vr = 8 * (i / (D / 64)) + (lane >> 3);
    const int vch = 8 * (i % (D / 64)) + ((lane & 7) ^ (2 * (lane >> 4)));
    koff[i] = uint32_t(kr * 2 * D + 16 * kch) + (kSpan - 1024u * i);
    voff[i] = uint32_t(vr * 2 * D + 16 * vch) + (kSpan - 1024u * i);
  }
  const int slot_mask = (1 << b.page_shift) - 1;
  const char* kp = static_cast<const char*>(t.k_pages);
  const char* vp = static_cast<const char*>(t.v_pages);
  // byte offset in the pool of the 16 keys from key j, which lie in page `page`
  auto half_offset = [&](int page, int j) __attribute__((always_inline)) {
    return ((int64_t(max(page, 0)) * b.kv_heads + head) * (slot_mask + 1) + (j & slot_mask)) * (2 * D);
  };

  // Copy block tb, whose halves lie in the given pages (a hole reads page 0: masked).
  auto fetch = [&](int tb, int page0, int page1) __attribute__((always_inline)) {
    constexpr int64_t kSpan = 1024 * (C::N - 1);
    const int j = blocks.key0(tb);
    const uint32_t dst = uint32_t(size_t(LDS_PTR(char, kbuf)));
    const int64_t a = uniform(half_offset(page0, j) - kSpan), c = uniform(half_offset(page1, j + 16) - kSpan);
    paged_copy<C::N, NT>(dst, kp + a, koff);
    paged_copy<C::N, NT>(dst + C::HALF, kp + c, koff);
    paged_copy<C::N, NT>(dst + C::BLOCK, vp + a, voff);
    paged_copy<C::N, NT>(dst + C::BLOCK + C::HALF, vp + c, voff);
  };

  // The wave's blocks.  A wave whose O is not finite goes over them again, with a reference so
  // far above the scores that its weights sum to at most 1: O then stays below the largest
  // |V|, and is not finite where a V element is not.  The rests of the probabilities meet such
  // an element as 0 or a negative number, which would make an infinity NaN: a third run leaves
  // them out.
  for (int run = 0;; ++run) {
    const bool rests = run < 2;
    const float raise = run == 0 ? kRaise : 0.0f;
    const float lift = run == 0 ? 0.0f : float(32 - __builtin_clz(uint32_t(kBK * (t1 - t0) | 1)));
#pragma unroll
    for (int x = 0; x < QT; ++x) {
      m_run[x] = -FLT_MAX;   // (finite: keys that score -inf get weight 0)
      l_run[x] = 0.0f;       // this lane's share of the sum of the probabilities
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt) o[dt][x] = f32x4{};
    }
    int tb = t0 + wave, i = 0;       // this wave's i-th block
    int page[2] = {-1, -1};
    if (tb < t1) {
      load_pages(0);
      page[0] = __builtin_amdgcn_readlane(page_of, 0);
      page[1] = __builtin_amdgcn_readlane(page_of, 1);
      fetch(tb, page[0], page[1]);
    }
    while (tb < t1) {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
      asm volatile("" ::: "memory");
      bf16x8 kc[2][C::KS];
      u32x4 va[C::DT];
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int ks = 0; ks < C::KS; ++ks)
          kc[kh][ks] = *reinterpret_cast<const bf16x8*>(kbuf + k_lane + 1024 * (kh * C::KS + ks));
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt) {
        const char* vt = vbuf + v_lane[dt % 4] + 1024 * (dt / 4);
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, vt));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, vt + 32 * D));
        const u32x2 lo2 = __builtin_bit_cast(u32x2, lo), hi2 = __builtin_bit_cast(u32x2, hi);
        va[dt] = u32x4{lo2[0], lo2[1], hi2[0], hi2[1]};
      }
      __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0): the reads are done
      __builtin_amdgcn_sched_barrier(0);
      const int j0 = blocks.key0(tb);
      const int cur[2] = {page[0], page[1]};
      const int next = tb + kWaves;
      ++i;
      if (next < t1) {
        if ((i & 31) == 0) load_pages(i);
        page[0] = __builtin_amdgcn_readlane(page_of, 2 * (i & 31));
        page[1] = __builtin_amdgcn_readlane(page_of, 2 * (i & 31) + 1);
        fetch(next, page[0], page[1]);
      }
      __builtin_amdgcn_sched_barrier(0);

      f32x4 s[2][QT];
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
          for (int x = 0; x < QT; ++x)
            s[kh][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kc[kh][ks], qreg[x][ks],
                                                               ks == 0 ? f32x4{} : s[kh][x], 0, 0, 0);

      // the block holds keys that some row does not see
      const bool edge = j0 + kBK > head_r.hi || cur[0] < 0 || cur[1] < 0 ||
                        (j0 < tail_r.lo && j0 + kBK > b.anchor_tokens);
      bool spread = false;   // some V element that is not finite was kept out of the products
      if (edge) {
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = j0 + 16 * kh + 4 * grp + e;
#pragma unroll
            for (int x = 0; x < QT; ++x) {
              const bool seen = cur[kh] >= 0 && j < see[x].hi && (j >= see[x].lo || j < b.anchor_tokens);
              s[kh][x][e] = seen ? s[kh][x][e] : -INFINITY;
            }
            // (a key some row may see: before the last row's end, behind the first row's start)
            const bool any = cur[kh] >= 0 && j < tail_r.hi && (j >= head_r.lo || j < b.anchor_tokens);
            if (!any)
#pragma unroll
              for (int dt = 0; dt < C::DT; ++dt)
                va[dt][2 * kh + (e >> 1)] &= (e & 1) ? 0x0000ffffu : 0xffff0000u;
          }
        if (rows_differ) {
          bool bad = false;
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int w = 0; w < 4; ++w) bad |= bf16_pair_not_finite(va[dt][w]);
          spread = __builtin_amdgcn_ballot_w64(bad) != 0;
          if (spread)
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
              for (int w = 0; w < 4; ++w) va[dt][w] = bf16_pair_finite(va[dt][w]);
        }
      }

      float mx[QT];
      bool over = false;
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        mx[x] = fmaxf(fmaxf(s[0][x][0], s[0][x][1]), fmaxf(s[0][x][2], s[0][x][3]));
        mx[x] = fmaxf(mx[x], fmaxf(fmaxf(s[1][x][0], s[1][x][1]), fmaxf(s[1][x][2], s[1][x][3])));
        mx[x] = fmaf(max_across_groups(mx[x]), t.scale_log2, lift);
        // the first block's max (lifted) is the reference from then on, until a score passes it far
        over |= mx[x] > (m_run[x] == -FLT_MAX ? m_run[x] : m_run[x] + raise);
      }
      if (__builtin_amdgcn_ballot_w64(over) != 0) {
#pragma unroll
        for (int x = 0; x < QT; ++x) {
          const float m_new = mx[x] > (m_run[x] == -FLT_MAX ? m_run[x] : m_run[x] + raise) ? mx[x] : m_run[x];
          const float alpha = __builtin_amdgcn_exp2f(m_run[x] - m_new);
          l_run[x] *= alpha;
          m_run[x] = m_new;
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[dt][x][e] *= alpha;
        }
      }
      uint32_t pk[QT][4], pr[QT][4];   // rounded, and the rests
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        float lb = 0.0f;
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kh][x][e], t.scale_log2, -m_run[x]));
            const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kh][x][e + 1], t.scale_log2, -m_run[x]));
            const uint32_t w = pack_bf16(p0, p1);
            pk[x][2 * kh + (e >> 1)] = w;
            pr[x][2 * kh + (e >> 1)] = pack_bf16(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u));
            lb += p0 + p1;
          }
        l_run[x] += lb;
      }
#pragma unroll
      for (int x = 0; x < QT; ++x) {
        const u32x4 pu = {pk[x][0], pk[x][1], pk[x][2], pk[x][3]}, ru = {pr[x][0], pr[x][1], pr[x][2], pr[x][3]};
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt) {
          const bf16x8 v = __builtin_bit_cast(bf16x8, va[dt]);
          o[dt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, pu), o[dt][x], 0, 0, 0);
          if (rests)
            o[dt][x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, __builtin_bit_cast(bf16x8, ru), o[dt][x], 0, 0, 0);
        }
      }
      if (spread) {
        // V elements that are not finite, for the rows that see their key (from the pool:
        // the copy in LDS is the next block's by now)
#pragma unroll 1
        for (int kk = 0; kk < kBK; ++kk) {
          const int kh = kk >> 4, j = j0 + kk;
          if (cur[kh] < 0 || j >= tail_r.hi) continue;
          const __bf16* vr = reinterpret_cast<const __bf16*>(vp + half_offset(cur[kh], j));
#pragma unroll
          for (int x = 0; x < QT; ++x) {
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) w = e == (kk >> 1 & 1) + 2 * kh ? pk[x][e] : w;
            const uint32_t pw = uint32_t(__shfl(int(w), l16 + 16 * ((kk & 15) >> 2)));
            const float p = __uint_as_float((kk & 1) ? pw & 0xffff0000u : pw << 16);
            const bool seen = j < see[x].hi && (j >= see[x].lo || j < b.anchor_tokens);
#pragma unroll
            for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float v = float(vr[16 * dt + 4 * grp + e]);
                if (seen && !isfinite(v)) o[dt][x][e] += p * v;
              }
          }
        }
      }
      tb = next;
    }
    float any = 0.0f;
#pragma unroll
    for (int x = 0; x < QT; ++x)
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) any = fmaf(o[dt][x][e], 0.0f, any);
    if (!rests || __builtin_amdgcn_ballot_w64(any != 0.0f) == 0) break;
  }

  // join the waves (over the K and V blocks, once all are read)
  __syncthreads();
  float* part = reinterpret_cast<float*>(lds);
  float* part_m = part + kWaves * C::kRows * C::kPitch;
  float* part_l = part_m + kWaves * C::kRows;
#pragma unroll
  for (int x = 0; x < QT; ++x) {
    const int row = wave * C::kRows + 16 * x + l16;
    const float l = sum_across_groups(l_run[x]);
    if (grp == 0) {
      part_m[row] = m_run[x];
      part_l[row] = l;
    }
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
      *reinterpret_cast<f32x4*>(part + row * C::kPitch + 16 * dt + 4 * grp) = o[dt][x];
  }
  __syncthreads();
  float* ws = t.part + (int64_t(item) * b.kv_heads + head) * paged_part_floats(C::kRows, D);
  for (int n = threadIdx.x; n < C::kRows * (D / 8); n += kThreads) {
    const int r = n / (D / 8), c = n % (D / 8);
    if (row0 + r > row1) continue;
    float m = part_m[r];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) m = fmaxf(m, part_m[w * C::kRows + r]);
    float l = 0.0f, a[kWaves];
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      a[w] = __builtin_amdgcn_exp2f(part_m[w * C::kRows + r] - m);
      l += a[w] * part_l[w * C::kRows + r];
    }
    const float inv = paged_inverse(l);
    f32x4 acc[2] = {};
    if (l != 0.0f)   // (a row that saw nothing is zero)
#pragma unroll
      for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          acc[x] += (a[w] * inv) * *reinterpret_cast<const f32x4*>(part + (w * C::kRows + r) * C::kPitch + 8 * c + 4 * x);
    if (it.parts > 1) {
      *reinterpret_cast<f32x4*>(ws + r * D + 8 * c) = acc[0];
      *reinterpret_cast<f32x4*>(ws + r * D + 8 * c + 4) = acc[1];
      if (c == 0) {
        ws[C::kRows * D + r] = m;
        ws[C::kRows * D + C::kRows + r] = l;
      }
    } else {
      const int tau = paged_token(b, row0 + r);
      const int64_t at = int64_t(it.seq.q0 + tau) * (b.kv_heads * b.group) + head * b.group +
                         (row0 + r - tau * b.group);
      paged_store<__bf16, 8>(static_cast<__bf16*>(t.out) + at * D + 8 * c, reinterpret_cast<const float*>(acc));
      if (t.lse != nullptr && c == 0) t.lse[at] = paged_lse(m, l);
    }
  }
}

// (tiles of 16 rows are chosen only where a sequence is one tile: once)
template <int D, int QT, int W>
hipError_t launch(bool once, const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                  int64_t items, hipStream_t stream) {
  const dim3 grid(unsigned(items * b.kv_heads));
  if (QT == 1 || once)
    hipLaunchKernelGGL((paged_attn_kernel<D, QT, W, true>), grid, dim3(64 * W), 0, stream, b, sp, t);
  else if constexpr (QT > 1)
    hipLaunchKernelGGL((paged_attn_kernel<D, QT, W, false>), grid, dim3(64 * W), 0, stream, b, sp, t);
  return hipGetLastError();
}

// Joins the parts of the tiles that have several: `slices` workgroups for each tile and kv
// head, which share the tile's outputs (rows by groups of four elements); inside a
// workgroup groups of threads share the parts, four in flight per thread, and join through
// LDS.  Bound by latency: a few loads deep, whatever the number of parts.
constexpr int kJoinThreads = 256;

template <class T, int D, int RT, int KB>
__global__ __launch_bounds__(kJoinThreads) void paged_join_kernel(PagedBatch b, PagedSplit sp,
                                                                  PagedTensors t, int max_items,
                                                                  int slices) {
  __shared__ f32x4 acc_s[kJoinThreads];
  __shared__ float m_s[kJoinThreads], l_s[kJoinThreads];
  const int lane = threadIdx.x & 63;
  const int slice = blockIdx.x % slices, head = blockIdx.x / slices % b.kv_heads;
  PagedItem it;
  if (!PagedScan<RT, KB>(b, sp, lane).find(blockIdx.x / slices / b.kv_heads, true, &it)) return;
  if (it.parts <= 1 || it.item0 + it.parts > max_items) return;
  const int n_rows = min(it.seq.n_new * b.group - it.tile * RT, RT);
  const int64_t stride = paged_part_floats(RT, D);
  const float* p0 = t.part + (int64_t(it.item0) * b.kv_heads + head) * stride;
  const int64_t step = stride * b.kv_heads;   // from part to part
  // (references are in log2 units in the bf16 kernels, in natural units in the float32 one)
  constexpr float kUnit = sizeof(T) == 2 ? 1.0f : 1.44269504f;

  const int outs = n_rows * (D / 4);                      // of the tile
  const int first = int(int64_t(slice) * outs / slices), end = int(int64_t(slice + 1) * outs / slices);
  for (int base = first; base < end; base += kJoinThreads) {
    const int n = min(end - base, kJoinThreads);          // outputs of this round
    const int groups = min(kJoinThreads / n, (it.parts + 3) / 4);   // that share the parts
    const int g = threadIdx.x / n, i = base + threadIdx.x % n;
    const int r = i / (D / 4), c = i % (D / 4);
    float m = -FLT_MAX, l = 0.0f;
    f32x4 acc = {};
    if (g < groups)
      for (int p = g; p < it.parts; p += 4 * groups) {
        float pm[4], pl[4];
        f32x4 pa[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float* pp = p0 + min(p + k * groups, it.parts - 1) * step;
          pm[k] = pp[RT * D + r];
          pl[k] = pp[RT * D + RT + r];
          pa[k] = *reinterpret_cast<const f32x4*>(pp + r * D + 4 * c);
        }
        float m_new = m;
#pragma unroll
        for (int k = 0; k < 4; ++k) m_new = fmaxf(m_new, p + k * groups < it.parts ? pm[k] : m_new);
        const float before = l * __builtin_amdgcn_exp2f((m - m_new) * kUnit);
        l = before;
#pragma unroll
        for (int k = 0; k < 4; ++k) {   // pl becomes the part's weight
          pl[k] = p + k * groups < it.parts ? pl[k] * __builtin_amdgcn_exp2f((pm[k] - m_new) * kUnit) : 0.0f;
          l += pl[k];
        }
        const float inv = paged_inverse(l);
        acc *= before * inv;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if (p + k * groups >= it.parts) break;
          acc += (pl[k] * inv) * pa[k];
        }
        m = m_new;
      }
    if (groups > 1) {   // (uniform)
      m_s[threadIdx.x] = m;
      l_s[threadIdx.x] = l;
      acc_s[threadIdx.x] = acc;
      __syncthreads();
      if (g == 0) {
        for (int k = 1; k < groups; ++k) m = fmaxf(m, m_s[threadIdx.x + k * n]);
        l = 0.0f;
        for (int k = 0; k < groups; ++k)
          l += l_s[threadIdx.x + k * n] * __builtin_amdgcn_exp2f((m_s[threadIdx.x + k * n] - m) * kUnit);
        const float inv = paged_inverse(l);
        acc = f32x4{};
        for (int k = 0; k < groups; ++k) {
          const int x = threadIdx.x + k * n;
          acc += (l_s[x] * __builtin_amdgcn_exp2f((m_s[x] - m) * kUnit) * inv) * acc_s[x];
        }
      }
      __syncthreads();
    }
    if (g == 0) {
      const int row = it.tile * RT + r, tau = paged_token(b, row);
      const int64_t at = int64_t(it.seq.q0 + tau) * (b.kv_heads * b.group) + head * b.group +
                         (row - tau * b.group);
      paged_store<T, 4>(static_cast<T*>(t.out) + at * D + 4 * c, reinterpret_cast<const float*>(&acc));
      if (t.lse != nullptr && c == 0) t.lse[at] = paged_lse(m * kUnit, l);
    }
  }
}

}  // namespace

hipError_t launch_paged_attn_bf16(int qt, int waves, bool once, const PagedBatch& b,
                                  const PagedSplit& sp, const PagedTensors& t, int64_t items,
                                  int head_dim, hipStream_t stream) {
  auto pick = [&](auto d, auto q) {
    constexpr int D = decltype(d)::value, Q = decltype(q)::value;
    return waves == 2 ? launch<D, Q, 2>(once, b, sp, t, items, stream)
                      : launch<D, Q, 4>(once, b, sp, t, items, stream);
  };
  using std::integral_constant;
  if (head_dim == 64)
    return qt == 2 ? pick(integral_constant<int, 64>{}, integral_constant<int, 2>{})
                   : pick(integral_constant<int, 64>{}, integral_constant<int, 1>{});
  return qt == 2 ? pick(integral_constant<int, 128>{}, integral_constant<int, 2>{})
                 : pick(integral_constant<int, 128>{}, integral_constant<int, 1>{});
}

hipError_t launch_paged_join(int rows, int used, const PagedBatch& b, const PagedSplit& sp,
                             const PagedTensors& t, int64_t items, int64_t tiles, int head_dim,
                             int dtype, hipStream_t stream) {
  // a workgroup for every 16 outputs of four elements, whose parts 16 groups of threads share
  // (one sequence of 12800 tokens, one head: 20.0 us in all with 2 outputs and as many groups
  // as fit, 14.9 with 16, 15.5 with 32), up to two per CU, four for the 256-row tiles (12
  // sequences of 25 rows, 8 heads: 32.3 us with two, 34.3 with eight, since each workgroup looks
  // its tile up)
  const int64_t groups = tiles * b.kv_heads;
  int64_t slices = (int64_t(used) * head_dim / 4 + 15) / 16;
  const int64_t most = ((rows > 32 ? 4 : 2) * device_cus() + groups - 1) / groups;
  slices = slices < most ? slices : most;
  const dim3 grid(unsigned(groups * slices));
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, grid, dim3(kJoinThreads), 0, stream, b, sp, t, int(items), int(slices));
    return hipGetLastError();
  };
  if (dtype == FF_DT_BF16) {
    if (rows == kPagedPromptRows)
      return head_dim == 64 ? go(paged_join_kernel<__bf16, 64, kPagedPromptRows, 64>)
                            : go(paged_join_kernel<__bf16, 128, kPagedPromptRows, 64>);
    if (head_dim == 64)
      return rows == 32 ? go(paged_join_kernel<__bf16, 64, 32, 32>) : go(paged_join_kernel<__bf16, 64, 16, 32>);
    return rows == 32 ? go(paged_join_kernel<__bf16, 128, 32, 32>) : go(paged_join_kernel<__bf16, 128, 16, 32>);
  }
  if (head_dim == 64)
    return rows == 32 ? go(paged_join_kernel<float, 64, 32, 16>) : go(paged_join_kernel<float, 64, 16, 16>);
  return rows == 32 ? go(paged_join_kernel<float, 128, 32, 16>) : go(paged_join_kernel<float, 128, 16, 16>);
}

}  // namespace ff
