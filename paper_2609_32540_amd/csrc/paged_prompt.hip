// Attention of many new tokens per sequence over a paged cache (prompts, slices of them,
// renderer chunks), bf16: the pipeline of attn_bf16.hip over tiles of rows and pages.
//
// Work split.  A tile is 256 rows (token, query head of the group) of one sequence and kv
// head, a workgroup of eight waves, one per CU; each wave owns 32 rows.  Where a batch has
// fewer tiles than the GPU has CUs, their keys are cut into parts (paged_plan.h), whose
// float32 partials paged_join_kernel joins.  The matrix unit bounds it.
//
// What differs from attn_bf16.hip:
//   keys     64-key tiles from the sequence's start (anchors, then the window or all), a
//            copying wave taking 16 of them, which lie in one page, from a base of its own.
//            The pages of 64 tiles sit in lane registers, with a bit per 16 keys for holes.
//   masks    rows see different keys: a wave masks the tiles that hold keys which one of its
//            rows does not see (one compare per score), and only those.
//   V        rows that no row of the workgroup sees are zeroed in LDS, whatever they held, a
//            tile ahead of their use; where rows see different keys, elements that are not
//            finite too, which are added to the rows that see them at the end (their weight
//            is positive: an infinity stays one).
//   passes   the fast pass needs a first block (32 keys) that every row sees a key of, which a
//            causal window does not give: those, and calls that want the log-sum-exp (the sum
//            of the unrounded probabilities), run the checked pass at once.  Where holes cover
//            the first block, or a block's window without anchors begins behind it in its tile,
//            a workgroup runs both (two prompts with such holes 633 us).
//   rounding probabilities as one bf16: a second product for their rests would cost half of the
//            products again.  The fast pass divides by the sum of the rounded values, as there,
//            the checked pass by that of the unrounded ones.
//   range    O stays below the largest |V| in the checked pass, whose weights sum to at most 1;
//            a fast pass that leaves float32's range is run again.
//
// Measured (32/8 heads x 128).  Prompts of 5003 and 3966 tokens, causal: 346 us = 1060 TFLOP/s
// of the visible pairs, 370 in the checked pass; 16384 tokens as one block 1300 TFLOP/s.  40
// heads, 4680 queries over 28080 keys 2.36 ms, 2.22 with pages of 64 tokens (attn_bf16.hip over
// a ring 2.35).  A 64-key step takes 1.7 us, a tile about 14 us beside its steps: workgroup
// launch, lookup and Q 7.5, the pages and the first copies 6.5, which nothing covers, as all of
// a CU's LDS is one workgroup's.

#include <hip/hip_runtime.h>

#include <float.h>
#include <math.h>

#include <utility>

#include "ff_paged_internal.h"

namespace ff {
namespace {

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kQH = 2;                      // 16-row halves per wave
constexpr int kWaveQ = 16 * kQH;            // rows per wave
constexpr int kBlockQ = kPagedPromptRows;   // rows per workgroup
static_assert(kBlockQ == kWaves * kWaveQ, "a tile is one workgroup");
constexpr int kBK = 64;                     // keys per tile
constexpr int kXcds = 8;
constexpr float kSumLimit = 16.0f;          // checked pass: largest sum of a lane's 8 probabilities of a
                                            // block that is kept, in units of 2^-lift
constexpr float kFastLimit = 0x1p64f;       // fast pass: largest row sum before the checked pass
// passes of the key loop
constexpr int kPassFast = 0;                // fixed reference, row sums of the rounded P on the matrix core
constexpr int kPassChecked = 2;             // reference raised per block (check_blk)
constexpr int kVReadsFirst = 0;             // V reads issued ahead of the first S^T product
constexpr int kHalfVALU = 20;               // plain VALU of a row half: 8 fma + 8 add + 4 packs
constexpr int kHalfVALUFast = 16;           // the fast pass: 8 fma + 4 packs and slack
constexpr int kCopyWaves = kWaves / 2;      // waves 0-3, the older one of each SIMD, copy the tiles

template <int D>
struct Cfg {
  static constexpr int KS = D / 32;          // 32-wide d slices of S^T = K Q^T
  static constexpr int DT = D / 16;          // 16-row d tiles of O^T
  static constexpr int ROWB = 2 * D;         // bytes per K/V row in LDS
  static constexpr int CPR = D / 8;          // 16-byte chunks per row
  static constexpr int RPB = 1024 / ROWB;    // rows per 1 KB wave copy
  static constexpr int BLOCKS = kBK / RPB;   // 1 KB copies per tile (per tensor)
  static constexpr int BLOCKS_PER_WAVE = BLOCKS / kCopyWaves;   // copies by waves 0 .. kCopyWaves-1
  static constexpr int TILE = kBK * ROWB;    // bytes of one K (or V) tile
  static constexpr int SLOT = 2 * TILE;      // K tile then V tile
  static constexpr int VGB = D / 64;         // 1 KB blocks per 8-row group of a V tile
  static constexpr int KGB = D / 32;         // 1 KB blocks per 16-row group of a K tile
  static_assert(BLOCKS % kCopyWaves == 0, "every copying wave copies the same number of 1 KB blocks");
};

// Instruction order of one half of a pipeline step, by sched_group_barrier
// classes (0x008 matrix, 0x100 LDS read, 0x002 VALU, 0x400 transcendental):
// NRF of the half's NR LDS reads and a few softmax instructions ahead of the
// first product, then NM products, the first NR - NRF of them each followed by
// one more LDS read, and all of them by their share of the softmax of one query
// half (NV plain VALU instructions: 8 fma, 8 add, 4 packs and some slack; 8
// exponentials).
template <int NM, int NR, int NRF, int NV, int NT, int I>
__device__ __forceinline__ void interleave_one() {
  __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
  if constexpr (I < NR - NRF) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  constexpr int v = (NV * (I + 1)) / NM - (NV * I) / NM;
  if constexpr (v > 0) __builtin_amdgcn_sched_group_barrier(0x002, v, 0);
  constexpr int t = (NT * (I + 1)) / NM - (NT * I) / NM;
  if constexpr (t > 0) __builtin_amdgcn_sched_group_barrier(0x400, t, 0);
}

template <int NM, int NR, int NRF, int NV, int NT, int... I>
__device__ __forceinline__ void interleave_seq(std::integer_sequence<int, I...>) {
  (interleave_one<NM, NR, NRF, NV, NT, I>(), ...);
}

template <int NM, int NR, int NRF, int NV>
__device__ __forceinline__ void interleave_half() {
  static_assert(NR - NRF <= NM, "every spread LDS read follows its own product");
  constexpr int kHead = 2, kHeadT = 1;
  if constexpr (NRF > 0) __builtin_amdgcn_sched_group_barrier(0x100, NRF, 0);
  __builtin_amdgcn_sched_group_barrier(0x002, kHead, 0);
  __builtin_amdgcn_sched_group_barrier(0x400, kHeadT, 0);
  interleave_seq<NM, NR, NRF, NV - kHead, 8 - kHeadT>(std::make_integer_sequence<int, NM>{});
}

template <int D>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
void paged_prompt_kernel(PagedBatch b, PagedSplit sp, PagedTensors t) {
  using C = Cfg<D>;
  __shared__ __attribute__((aligned(1024))) char lds[5 * C::SLOT];
  auto slot = [&](int i) __attribute__((always_inline)) { return lds + i * C::SLOT; };
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);   // uniform
  const int lane = tid & 63;
  const int l16 = lane & 15;
  const int grp = lane >> 4;

  // Workgroup bx runs on XCD bx % 8.  Heads are dealt to the XCDs round robin, whole (a head's
  // tiles share its keys in one L2; the last kv_heads % 8 heads run in order), and a head's
  // last items come first: in a causal sequence they are the longest.  The grid is sized for
  // any batch of as many rows; the workgroups it has too many come last: an XCD deals its
  // workgroups to its engines in turn whether they have work or not (with two of 21 items
  // per head empty, 40 heads x 128, 4680 queries over 28080 keys took 2.8 instead of 2.4 ms).
  const PagedScan<kBlockQ, kBK> scan(b, sp, lane);
  const int n_items = gridDim.x / b.kv_heads;
  const int n_used = min(scan.count(), n_items);
  int head, item;
  {
    const int even = b.kv_heads - b.kv_heads % kXcds;
    const bool whole = blockIdx.x < unsigned(even * n_items);
    const int i = whole ? blockIdx.x / kXcds : blockIdx.x - even * n_items;
    if (i >= n_used * (whole ? even / kXcds : b.kv_heads - even)) return;
    head = whole ? blockIdx.x % kXcds + kXcds * (i / n_used) : even + i / n_used;
    item = n_used - 1 - i % n_used;
  }
  PagedItem it;
  if (!scan.find(item, false, &it)) return;
  const int n_rows = it.seq.n_new * b.group;
  const int row0 = it.tile * kBlockQ;
  const int row1 = min(row0 + kBlockQ, n_rows) - 1;
  const PagedRange head_r = paged_range(b, it.seq, paged_token(b, row0));    // first and last row
  const PagedRange tail_r = paged_range(b, it.seq, paged_token(b, row1));
  const bool rows_differ = head_r.hi != tail_r.hi || head_r.lo != tail_r.lo;
  const PagedBlocks<kBK> blocks = paged_blocks<kBK>(b, head_r, tail_r);
  const int t_begin = uniform(int(int64_t(it.part) * blocks.n / it.parts));
  const int n_tiles = uniform(int(int64_t(it.part + 1) * blocks.n / it.parts)) - t_begin;

  // Q^T operand: lane (l16, grp) of row half qh holds row q0 + 16 qh + l16, elements
  // d = 32 s + 8 grp .. +7 of slice s; hi and lo bound the keys that the row sees.
  const int q0 = row0 + wave * kWaveQ;
  const bool idle = q0 > row1;   // no rows for this wave: it only copies and keeps the barriers
  bf16x8 qreg[kQH][C::KS];
  int hi[kQH], lo[kQH];
#pragma unroll
  for (int qh = 0; qh < kQH; ++qh) {
    const int r = min(q0 + 16 * qh + l16, row1);
    const int tau = paged_token(b, r);
    const PagedRange see = paged_range(b, it.seq, tau);
    hi[qh] = see.hi;
    lo[qh] = see.lo;
    const __bf16* qp = static_cast<const __bf16*>(t.q) + int64_t(it.seq.q0 + tau) * t.q_stride +
                       int64_t(head * b.group + r - tau * b.group) * D + 8 * grp;
#pragma unroll
    for (int s = 0; s < C::KS; ++s) qreg[qh][s] = *reinterpret_cast<const bf16x8*>(qp + 32 * s);
  }
  // this wave's first and last row
  const PagedRange first_r = paged_range(b, it.seq, paged_token(b, min(q0, row1)));
  const PagedRange last_r = paged_range(b, it.seq, paged_token(b, min(q0 + kWaveQ - 1, row1)));

  // O^T tile (d tile dt, row half qh): lane (l16, grp) holds row q0 + 16 qh + l16 at
  // d = 16 dt + 4 grp + j, j = 0 .. 3
  f32x4 o[C::DT][kQH];
#pragma unroll
  for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh) o[dt][qh] = f32x4{};
  float m_run[kQH], l_run[kQH];
  f32x4 lsum[kQH];          // fast pass: row sums (every row of the tile holds the sum)
#pragma unroll
  for (int qh = 0; qh < kQH; ++qh) {
    m_run[qh] = -FLT_MAX;   // reference max of the scaled logits (log2 units)
    l_run[qh] = 0.0f;       // checked pass: this lane's partial sum of probabilities
    lsum[qh] = f32x4{};
  }

  // Pages of 64 tiles: lane l holds, of tile n0 + l, the page of this wave's 16 keys (waves
  // 0-3, which copy) and a bit for each 16 keys that are in a hole or behind the sequence's end.
  int tp = 0, th = 0;
  auto load_pages = [&](int n0) __attribute__((always_inline)) {
    int own = 0, bits = 0;
    if (n0 + lane < n_tiles) {
      const int k0 = blocks.key0(t_begin + n0 + lane);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int p = k0 + 16 * g < it.seq.keys ? paged_page(b, it.s, k0 + 16 * g) : -1;
        if (p < 0) bits |= 1 << g;
        if (g == (wave & 3)) own = max(p, 0);
      }
    }
    tp = own;
    th = bits;
  };

  // Copy of tile n into the slot at base (layouts as in attn_bf16.hip: K chunk-major per 16
  // keys, V d-blocked per 8), 16 keys per copying wave; holes read page 0.  Returns the
  // tile's hole bits.
  const int page_mask = (1 << b.page_shift) - 1;
  auto issue_tile = [&](char* base, int n) __attribute__((always_inline)) {
    if ((n & 63) == 0) load_pages(n);
    const int bits = __builtin_amdgcn_readlane(th, n & 63);
    if (wave < kCopyWaves) {
      constexpr int N = C::BLOCKS_PER_WAVE;
      constexpr uint32_t kSpan = 1024u * (N - 1);   // largest immediate offset
      int ln = lane;
      asm volatile("" : "+v"(ln));
      const int64_t page = __builtin_amdgcn_readlane(tp, n & 63);
      const int k0 = blocks.key0(t_begin + n) + 16 * wave;
      const int64_t off = uniform(((page * b.kv_heads + head) * (page_mask + 1) + (k0 & page_mask)) * C::ROWB - kSpan);
      uint32_t koff[N], voff[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int kr = ln & 15, kch = 4 * i + (ln >> 4);
        const int vr = 8 * (i / C::VGB) + ((ln & 15) >> 1);
        const int vch = 8 * (i % C::VGB) + 2 * (ln >> 4) + (ln & 1);
        koff[i] = uint32_t(kr * C::ROWB + 16 * kch) + (kSpan - 1024u * i);
        voff[i] = uint32_t(vr * C::ROWB + 16 * vch) + (kSpan - 1024u * i);
      }
      const uint32_t dst = uint32_t(size_t(LDS_PTR(char, base))) + wave * N * 1024;
      lds_copy_blocks<N>(dst, static_cast<const char*>(t.k_pages) + off, koff);
      lds_copy_blocks<N>(dst + C::TILE, static_cast<const char*>(t.v_pages) + off, voff);
    }
    return bits;
  };
  // keys k0 .. k0 + 63 include one that some row between those of ranges a and z does not see
  auto edge = [&](const PagedRange& a, const PagedRange& z, int k0, int bits) __attribute__((always_inline)) {
    return bits != 0 || k0 + kBK > a.hi || (k0 < z.lo && k0 + kBK > b.anchor_tokens);
  };
  // V rows of the tile at vt (first key k0) that no row of the workgroup sees become zero, and
  // where rows see different keys elements that are not finite; wave w has rows 8 w .. 8 w + 7.
  // The fast pass does this for tiles that hold places of no token, whose memory may hold
  // anything; tokens that are not finite are left to show in its sums (see below).
  bool bad = false;
  auto must_clean = [&](int k0, int bits, auto pass) __attribute__((always_inline)) {
    if constexpr (decltype(pass)::value == kPassFast) return bits != 0 || k0 + kBK > it.seq.keys;
    else return edge(head_r, tail_r, k0, bits);
  };
  auto clean_v = [&](char* vt, int k0, int bits) {
#pragma unroll
    for (int c = 0; c < 8 * C::ROWB / 1024; ++c) {
      const int off = 1024 * c + 16 * lane;
      const int key = k0 + 8 * wave + ((off & 255) >> 5);
      const bool any = ((bits >> (wave >> 1)) & 1) == 0 && key < tail_r.hi &&
                       (key >= head_r.lo || key < b.anchor_tokens);
      u32x4* p = reinterpret_cast<u32x4*>(vt + 8 * C::ROWB * wave + off);
      if (!any) {
        *p = u32x4{};
      } else if (rows_differ) {
        u32x4 x = *p;
        bool found = false;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          found |= bf16_pair_not_finite(x[w]);
          x[w] = bf16_pair_finite(x[w]);
        }
        if (found) *p = x;
        bad |= found;
      }
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // written before the next barrier
  };

  // LDS read addresses.  The swizzle only flips chunk bits that the row offset
  // leaves clear, so each read is (slot + immediate) + (lane base ^ constant):
  //   K (A of S^T), row 16 kh + l16, chunk 4 ks + grp: k_lane + 1024 ks + 16 ROWB kh
  //     in the chunk-major K tile (a 16-lane quarter reads one whole 256-byte line);
  //   V (A of O^T, transposing read), lane group grp reads key rows 4 grp .. 4 grp+3
  //     (lo) and 16 + 4 grp .. +3 (hi) of the block, lane l16 the row 4 grp + l16 / 4
  //     (+ 16) at d offset 4 (l16 % 4) of the d tile, and receives column l16 of the
  //     four rows: v_lane[lo/hi] + 256 dt for d tile dt in the d-blocked V tile
  //     (a 32-lane half reads one whole 256-byte line: no bank conflicts).
  const int k_lane = 256 * grp + 16 * l16;
  int v_lane[2];
#pragma unroll
  for (int hi = 0; hi < 2; ++hi) {
    const int r = 16 * hi + 4 * grp + (l16 >> 2);
    v_lane[hi] = (r >> 3) * (8 * C::ROWB) + ((2 * (r & 7) + ((l16 >> 1) & 1)) << 4) + 8 * (l16 & 1);
  }

  // K operands of S^T for 32-key block kb of the tile at kt: a[kh][ks] = rows
  // 16 kh + l16, d slice ks
  auto k_read = [&](const char* kt, int kb, bf16x8 (&a)[2][C::KS]) __attribute__((always_inline)) {
    const char* kbase = kt + kb * 32 * C::ROWB;
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks)
        a[kh][ks] = *reinterpret_cast<const bf16x8*>(kbase + kh * 16 * C::ROWB + k_lane + 1024 * ks);
  };
  // S^T of a block: tile (kh, qh) = keys 16 kh .. +15 x queries 16 qh .. +15 of
  // the wave; lane (l16, grp) register j holds key 16 kh + 4 grp + j of query
  // 16 qh + l16
  auto s_mma = [&](const bf16x8 (&a)[2][C::KS], f32x4 (&s)[2][kQH]) __attribute__((always_inline)) {
#pragma unroll
    for (int ks = 0; ks < C::KS; ++ks)
#pragma unroll
      for (int kh = 0; kh < 2; ++kh)
#pragma unroll
        for (int qh = 0; qh < kQH; ++qh)
          s[kh][qh] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[kh][ks], qreg[qh][ks],
                                                              ks == 0 ? f32x4{} : s[kh][qh], 0, 0, 0);
  };
  // V^T operands of O^T for 32-key block kb of the tile at vt, d tile dt
  auto v_read = [&](const char* vt, int kb, bf16x8 (&a)[C::DT]) __attribute__((always_inline)) {
    const char* vbase = vt + kb * 32 * C::ROWB;
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt) {
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, vbase + v_lane[0] + 256 * dt));
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(s16x4, vbase + v_lane[1] + 256 * dt));
      const u32x2 lo2 = __builtin_bit_cast(u32x2, lo), hi2 = __builtin_bit_cast(u32x2, hi);
      const u32x4 au = {lo2[0], lo2[1], hi2[0], hi2[1]};
      a[dt] = __builtin_bit_cast(bf16x8, au);
    }
  };
  // O^T += V^T P^T for one block; with_sums also adds the block's row sums into
  // lsum (an all-ones A operand: every row of the 16 x 16 result is the column
  // sum of P^T, i.e. the sum of exactly the rounded probabilities O^T adds up)
  auto pv_mma = [&](const bf16x8 (&a)[C::DT], const uint32_t (&pk)[kQH][4], auto with_sums)
      __attribute__((always_inline)) {
    bf16x8 pb[kQH];
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh) {
      const u32x4 pu = {pk[qh][0], pk[qh][1], pk[qh][2], pk[qh][3]};
      pb[qh] = __builtin_bit_cast(bf16x8, pu);
    }
#pragma unroll
    for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
      for (int qh = 0; qh < kQH; ++qh)
        o[dt][qh] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[dt], pb[qh], o[dt][qh], 0, 0, 0);
    if constexpr (decltype(with_sums)::value) {
      const bf16x8 ones = {__bf16(1.0f), __bf16(1.0f), __bf16(1.0f), __bf16(1.0f),
                           __bf16(1.0f), __bf16(1.0f), __bf16(1.0f), __bf16(1.0f)};
#pragma unroll
      for (int qh = 0; qh < kQH; ++qh)
        lsum[qh] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pb[qh], lsum[qh], 0, 0, 0);
    }
  };
  // mask the keys of a 32-key block from key j0 that a row does not see (bits: its holes)
  const bool only_hi = last_r.lo == 0;   // every row of the wave sees all keys before its own end
  auto mask_blk = [&](f32x4 (&s)[2][kQH], int j0, int bits) __attribute__((always_inline)) {
    if (only_hi && bits == 0) {
#pragma unroll
      for (int qh = 0; qh < kQH; ++qh) {
        const int n = hi[qh] - j0 - 4 * grp;
#pragma unroll
        for (int kh = 0; kh < 2; ++kh)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[kh][qh][j] = 16 * kh + j < n ? s[kh][qh][j] : -INFINITY;
      }
      return;
    }
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = j0 + 16 * kh + 4 * grp + j;
        const bool there = ((bits >> kh) & 1) == 0;
#pragma unroll
        for (int qh = 0; qh < kQH; ++qh) {
          const bool seen = there && key < hi[qh] && (key >= lo[qh] || key < b.anchor_tokens);
          s[kh][qh][j] = seen ? s[kh][qh][j] : -INFINITY;
        }
      }
  };
  // column max of a block for query half qh (every lane of the query agrees)
  auto col_max = [&](const f32x4 (&s)[2][kQH], int qh) __attribute__((always_inline)) {
    float mx = fmaxf(fmaxf(s[0][qh][0], s[0][qh][1]), fmaxf(s[0][qh][2], s[0][qh][3]));
    mx = fmaxf(mx, fmaxf(fmaxf(s[1][qh][0], s[1][qh][1]), fmaxf(s[1][qh][2], s[1][qh][3])));
    return max_across_groups(mx);
  };
  // probabilities of query half qh of a block as packed bf16: pk[qh] is the
  // P^T operand of that half, keys 4 grp .. 4 grp+3 then 16 + 4 grp .. +3; with
  // with_sums, lb[qh] is this lane's share of the block's row sum
  auto p_half = [&](const f32x4 (&s)[2][kQH], int qh, uint32_t (&pk)[kQH][4], float (&lb)[kQH],
                    auto with_sums) __attribute__((always_inline)) {
    float sum = 0.0f;
#pragma unroll
    for (int kh = 0; kh < 2; ++kh)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[kh][qh][j], t.scale_log2, -m_run[qh]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(s[kh][qh][j + 1], t.scale_log2, -m_run[qh]));
        pk[qh][2 * kh + (j >> 1)] = pack_bf16(p0, p1);
        if constexpr (decltype(with_sums)::value) sum += p0 + p1;
      }
    if constexpr (decltype(with_sums)::value) lb[qh] = sum;
  };
  auto p_blk = [&](const f32x4 (&s)[2][kQH], uint32_t (&pk)[kQH][4], float (&lb)[kQH])
      __attribute__((always_inline)) {
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh) p_half(s, qh, pk, lb, std::true_type{});
  };
  // The reference is only raised when a lane's probabilities of a block (relative to
  // it) sum past the limit: then it is raised to the block's column max plus lift
  // (O and l follow) and the probabilities are redone from the scores, which
  // are still in registers.  Infinities (scores far above the reference) also
  // exceed the limit.  The lift makes all probabilities of a row sum to at most 1
  // (64 2^-lift from each block's four lanes), so that O stays below the largest
  // |V|.  O is rescaled after the products of the previous block (issued in the
  // same step) have been added into it.
  const int lift_bits = 6 + 32 - __builtin_clz(uint32_t(2 * n_tiles) | 1u);
  const float lift = float(lift_bits), sum_limit = __builtin_amdgcn_ldexpf(kSumLimit, -lift_bits);
  auto check_blk = [&](const f32x4 (&s)[2][kQH], uint32_t (&pk)[kQH][4], float (&lb)[kQH])
      __attribute__((always_inline)) {
    bool over = false;
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh) over |= lb[qh] > sum_limit;
    if (__builtin_amdgcn_ballot_w64(over) != 0) {
      float alpha[kQH];
#pragma unroll
      for (int qh = 0; qh < kQH; ++qh) {
        const float m_new = fmaxf(m_run[qh], fmaf(col_max(s, qh), t.scale_log2, lift));
        alpha[qh] = __builtin_amdgcn_exp2f(m_run[qh] - m_new);
        l_run[qh] *= alpha[qh];
        m_run[qh] = m_new;
      }
      p_blk(s, pk, lb);
      // O follows the raised reference only in the lanes whose reference moved
      if (alpha[0] != 1.0f || alpha[1] != 1.0f)
#pragma unroll
        for (int qh = 0; qh < kQH; ++qh)
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[dt][qh][j] *= alpha[qh];
    }
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh) l_run[qh] += lb[qh];
  };
  // One step of the block pipeline, in two halves that the scheduler may not
  // mix: (1) the V reads of this step, S^T of block b+1 from the K operands read
  // in the previous step and the softmax of query half 0 of block b; (2) the K
  // reads of the next step (tile kt_next, key block kb_next, into the registers
  // the S^T products have just consumed), O^T += P(b-1) V(b-1) and the softmax
  // of query half 1.  Inside a half every product is followed by its share of
  // the LDS reads and of the softmax work (exponentials, row sums, bf16
  // packing), which depends on no product of the step.  The fast pass sums
  // the probabilities on the matrix core, the checked pass with VALU adds
  // (its per-block check needs each block's sum).
  auto step = [&](bf16x8 (&ka)[2][C::KS], const char* vt, int kbv, const char* kt_next, int kb_next,
                  const f32x4 (&s_in)[2][kQH], f32x4 (&s_out)[2][kQH],
                  const uint32_t (&pk_in)[kQH][4], uint32_t (&pk_out)[kQH][4], float (&lb)[kQH],
                  auto pass) __attribute__((always_inline)) {
    constexpr bool kVSums = decltype(pass)::value != kPassFast;   // row sums in VALU
    constexpr int kNV = kVSums ? kHalfVALU : kHalfVALUFast;
    bf16x8 va[C::DT];
    v_read(vt, kbv, va);
    s_mma(ka, s_out);
    p_half(s_in, 0, pk_out, lb, std::bool_constant<kVSums>{});
    interleave_half<4 * C::KS, 2 * C::DT, kVReadsFirst, kNV>();
    __builtin_amdgcn_sched_barrier(0);
    k_read(kt_next, kb_next, ka);
    pv_mma(va, pk_in, std::bool_constant<!kVSums>{});
    p_half(s_in, 1, pk_out, lb, std::bool_constant<kVSums>{});
    interleave_half<2 * C::DT + (kVSums ? 0 : kQH), 2 * C::KS, 0, kNV>();
    // (the softmax results are computed inside this step, not sunk past the
    // branches that follow it)
    asm volatile("" ::"v"(pk_out[0][0]), "v"(pk_out[0][1]), "v"(pk_out[0][2]), "v"(pk_out[0][3]),
                 "v"(pk_out[1][0]), "v"(pk_out[1][1]), "v"(pk_out[1][2]), "v"(pk_out[1][3]));
    if constexpr (kVSums) asm volatile("" ::"v"(lb[0]), "v"(lb[1]));
    __builtin_amdgcn_sched_barrier(0);
  };

  auto key_loop = [&](auto pass) __attribute__((always_inline)) {
    constexpr int kPass = decltype(pass)::value;
    auto after_step = [&](const f32x4 (&s)[2][kQH], uint32_t (&pk)[kQH][4], float (&lb)[kQH])
        __attribute__((always_inline)) {
      if constexpr (kPass == kPassChecked) check_blk(s, pk, lb);
    };

    // ---- prologue: tiles 0 .. 2 in flight, S^T of block 0 ----------------------
    // Tile n lives in slot n % 5; bits0 .. bits2 are the hole bits of tiles n .. n + 2.
    int bits0 = issue_tile(slot(0), 0), bits1 = 0, bits2 = 0;
    if (n_tiles > 1) bits1 = issue_tile(slot(1), 1);
    if (n_tiles > 2) bits2 = issue_tile(slot(2), 2);
    int k0 = blocks.key0(t_begin);
    // the first step adds P = 0 times the V block of a tile -1: zeros
    for (int i = 16 * tid; i < C::TILE / 2; i += 16 * kThreads)
      *reinterpret_cast<u32x4*>(slot(4) + C::TILE + C::TILE / 2 + i) = u32x4{};
    // (tiles 1 and 2 may stay in flight)
    if (n_tiles > 2) __builtin_amdgcn_s_waitcnt(waitcnt_vm(4 * C::BLOCKS_PER_WAVE));
    else __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (must_clean(k0, bits0, pass)) {
      clean_v(slot(0) + C::TILE, k0, bits0);
      __syncthreads();
    }
    if (idle) {   // the copies, barriers and V rows of the loop below, no products
      int i1 = 1, i3 = 3;   // slots of tiles n + 1 and n + 3
#pragma unroll 1
      for (int n = 0; n < n_tiles; ++n) {
        if (wave < kCopyWaves) {
          if (n + 2 < n_tiles)
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * C::BLOCKS_PER_WAVE));
          else
            __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
        }
        asm volatile("s_barrier" ::: "memory");
        int bits3 = 0;
        if (n + 3 < n_tiles) bits3 = issue_tile(slot(i3), n + 3);
        if (n + 1 < n_tiles) {
          const int k1 = blocks.key0(t_begin + n + 1);
          if (must_clean(k1, bits1, pass)) clean_v(slot(i1) + C::TILE, k1, bits1);
        }
        bits1 = bits2;
        bits2 = bits3;
        i1 = i1 == 4 ? 0 : i1 + 1;
        i3 = i3 == 4 ? 0 : i3 + 1;
      }
      return;
    }
    // S^T of even blocks (block 0 of a tile) lives in s_a, of odd blocks in s_b;
    // P of even blocks in pk_a, of odd blocks in pk_b
    f32x4 s_a[2][kQH], s_b[2][kQH];
    uint32_t pk_a[kQH][4], pk_b[kQH][4];
    float lb[kQH];
    bf16x8 ka[2][C::KS];
    k_read(slot(0), 0, ka);
    s_mma(ka, s_a);
    k_read(slot(0), 1, ka);
    bool mask0 = edge(first_r, last_r, k0, bits0);   // tile n needs masks
    if (mask0) mask_blk(s_a, k0, bits0);
    // reference from the first block: its column max (O and l are zero), lifted in the
    // checked pass; finite, so that keys that score -inf and rows that see none of the
    // block get weight 0
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh)
      m_run[qh] = fmaxf(fmaf(col_max(s_a, qh), t.scale_log2, kPass == kPassChecked ? lift : 0.0f), -FLT_MAX);
#pragma unroll
    for (int qh = 0; qh < kQH; ++qh)
#pragma unroll
      for (int i = 0; i < 4; ++i) pk_b[qh][i] = 0;

    // ---- main loop over tiles: a barrier and two pipeline steps per tile -----
    // as in attn_bf16.hip; V of tile n + 1, first read after barrier n + 1, is cleaned
    // between the barriers
    int i0 = 0;   // slot of tile n
#pragma unroll 1
    for (int n = 0; n < n_tiles; ++n) {
      const int i1 = i0 == 4 ? 0 : i0 + 1;
      const int i4 = i0 == 0 ? 4 : i0 - 1;        // slot of tile n-1
      const int i3 = i0 >= 2 ? i0 - 2 : i0 + 3;   // slot of tile n-2 (and of tile n+3)
      if (wave < kCopyWaves) {
        if (n + 2 < n_tiles)
          __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * C::BLOCKS_PER_WAVE));
        else
          __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
      }
      asm volatile("s_barrier" ::: "memory");
      int bits3 = 0;
      if (n + 3 < n_tiles) bits3 = issue_tile(slot(i3), n + 3);
      char* st = slot(i0);
      char* sn = slot(i1);
      const int k1 = blocks.key0(t_begin + n + 1);
      bool mask1 = false;
      if (n + 1 < n_tiles) {
        mask1 = edge(first_r, last_r, k1, bits1);
        if (must_clean(k1, bits1, pass)) clean_v(sn + C::TILE, k1, bits1);
      }
      step(ka, slot(i4) + C::TILE, 1, sn, 0, s_a, s_b, pk_b, pk_a, lb, pass);
      if (mask0) mask_blk(s_b, k0 + 32, bits0 >> 2);
      after_step(s_a, pk_a, lb);
      step(ka, st + C::TILE, 0, sn, 1, s_b, s_a, pk_a, pk_b, lb, pass);
      if (mask1) mask_blk(s_a, k1, bits1);
      after_step(s_b, pk_b, lb);
      k0 = k1;
      mask0 = mask1;
      bits0 = bits1;
      bits1 = bits2;
      bits2 = bits3;
      i0 = i1;
    }
    {
      // O^T += P V of block 1 of the last tile
      bf16x8 va[C::DT];
      v_read(slot(i0 == 0 ? 4 : i0 - 1) + C::TILE, 1, va);
      pv_mma(va, pk_b, std::bool_constant<kPass == kPassFast>{});
    }
  };

  float l_tot[kQH];   // the row sum of the lane's row
#pragma unroll
  for (int qh = 0; qh < kQH; ++qh) l_tot[qh] = 0.0f;
  if (n_tiles > 0) {
    // One word per wave through LDS (the tiles are no longer read after the first barrier):
    // what any wave found.
    auto found = [&](bool overflow) __attribute__((always_inline)) {
      const int mine = (__builtin_amdgcn_ballot_w64(overflow) != 0 ? 1 : 0) |
                       (__builtin_amdgcn_ballot_w64(bad) != 0 ? 2 : 0);
      __builtin_amdgcn_s_waitcnt(0);
      __syncthreads();
      int* flags = reinterpret_cast<int*>(lds);
      if (lane == 0) flags[wave] = mine;
      __syncthreads();
      int all = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) all |= flags[w];
      return all;
    };
    bool checked_pass = t.lse != nullptr || (b.window >= 0 && !b.block);
    int all = 0;
    if (!checked_pass) {
      key_loop(std::integral_constant<int, kPassFast>{});
      bool overflow = false;
#pragma unroll
      for (int qh = 0; qh < kQH; ++qh) {
        l_tot[qh] = lsum[qh][0];
        overflow |= !(l_tot[qh] <= kFastLimit);   // (a NaN sum counts as an overflow)
        // a V element that is not finite has made its column of O so, for every row
        float any = 0.0f;
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
          for (int j = 0; j < 4; ++j) any = fmaf(o[dt][qh][j], 0.0f, any);
        overflow |= any != 0.0f;
      }
      all = found(overflow);
      checked_pass = (all & 1) != 0;
      if (checked_pass) {
        __syncthreads();   // (every wave has read the flags)
#pragma unroll
        for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
          for (int qh = 0; qh < kQH; ++qh) o[dt][qh] = f32x4{};
#pragma unroll
        for (int qh = 0; qh < kQH; ++qh) l_run[qh] = 0.0f;
        bad = false;
      }
    }
    if (checked_pass) {
      key_loop(std::integral_constant<int, kPassChecked>{});
#pragma unroll
      for (int qh = 0; qh < kQH; ++qh) l_tot[qh] = sum_across_groups(l_run[qh]);
      all = found(false);
    }

    // V elements that clean_v kept out of the products, for the rows that see their key
    if ((all & 2) != 0 && rows_differ) {
#pragma unroll 1
      for (int n = 0; n < kBK * n_tiles; ++n) {
        const int key = blocks.key0(t_begin + n / kBK) + n % kBK;
        if (key >= tail_r.hi) continue;
        const int64_t page = paged_page(b, it.s, key);
        if (page < 0) continue;
        const __bf16* vr = static_cast<const __bf16*>(t.v_pages) +
                           ((page * b.kv_heads + head) * (page_mask + 1) + (key & page_mask)) * D;
        const int k0 = key / kBK * kBK;
        // (a tile whose keys every row sees was left whole)
        int bits = 0;
        for (int g = 0; g < 4; ++g)
          if (k0 + 16 * g >= it.seq.keys || paged_page(b, it.s, k0 + 16 * g) < 0) bits |= 1 << g;
        if (!edge(head_r, tail_r, k0, bits)) continue;
#pragma unroll
        for (int qh = 0; qh < kQH; ++qh) {
          const bool seen = key < hi[qh] && (key >= lo[qh] || key < b.anchor_tokens);
#pragma unroll
          for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float v = float(vr[16 * dt + 4 * grp + j]);
              if (seen && !isfinite(v)) o[dt][qh][j] += v;
            }
        }
      }
    }
  }

  // normalise and store: lane (l16, grp) of tile (dt, qh) holds row q0 + 16 qh + l16 at
  // d = 16 dt + 4 grp + j
#pragma unroll
  for (int qh = 0; qh < kQH; ++qh) {
    const int r = q0 + 16 * qh + l16;
    // a row that saw nothing (l = 0) is zero
    const float inv = 1.0f / l_tot[qh];
    const bool some = l_tot[qh] != 0.0f;
    if (it.parts > 1) {
      if (r > row1) continue;
      float* ws = t.part + (int64_t(item) * b.kv_heads + head) * paged_part_floats(kBlockQ, D);
      const int row = r - row0;
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
        *reinterpret_cast<f32x4*>(ws + row * D + 16 * dt + 4 * grp) = some ? o[dt][qh] * inv : f32x4{};
      if (grp == 0) {
        ws[kBlockQ * D + row] = m_run[qh];
        ws[kBlockQ * D + kBlockQ + row] = l_tot[qh];
      }
    } else {
      uint32_t w[C::DT][2];
#pragma unroll
      for (int dt = 0; dt < C::DT; ++dt)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          w[dt][h] = some ? pack_bf16(o[dt][qh][2 * h] * inv, o[dt][qh][2 * h + 1] * inv) : 0u;
      const int tau = paged_token(b, min(r, row1));
      const int64_t at = int64_t(it.seq.q0 + tau) * (b.kv_heads * b.group) + head * b.group +
                         (min(r, row1) - tau * b.group);
      __bf16* op = static_cast<__bf16*>(t.out) + at * D + 8 * grp;
      // two d tiles, 8 bytes of each per lane, become 16 bytes in a row: lane group g takes
      // d = 32 k + 8 g .. +7
#pragma unroll
      for (int k = 0; k < C::DT / 2; ++k) {
        uint32_t lo[2], hi2[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          auto x = __builtin_amdgcn_permlane32_swap(w[2 * k][h], w[2 * k + 1][h], false, false);
          x = __builtin_amdgcn_permlane16_swap(x[0], x[1], false, false);
          lo[h] = x[0];
          hi2[h] = x[1];
        }
        if (r <= row1) *reinterpret_cast<u32x4*>(op + 32 * k) = u32x4{lo[0], lo[1], hi2[0], hi2[1]};
      }
      if (t.lse != nullptr && grp == 0 && r <= row1) t.lse[at] = paged_lse(m_run[qh], l_tot[qh]);
    }
  }
}

}  // namespace

hipError_t launch_paged_prompt(const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                               int64_t items, int head_dim, hipStream_t stream) {
  const dim3 grid(unsigned(items * b.kv_heads));
  if (head_dim == 128)
    hipLaunchKernelGGL(paged_prompt_kernel<128>, grid, dim3(kThreads), 0, stream, b, sp, t);
  else
    hipLaunchKernelGGL(paged_prompt_kernel<64>, grid, dim3(kThreads), 0, stream, b, sp, t);
  return hipGetLastError();
}

}  // namespace ff
