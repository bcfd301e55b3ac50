// What the kernels of the paged cache share: the batch as a launch passes it, the keys
// that a query sees, and the device-side division of a batch into work items.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_tile.h"

namespace ff {

// One batch over a page pool (include/ff_paged.h).  The arrays are the caller's, in
// device memory, and are not trusted: every index taken from them is brought into range
// (paged_seq) or tested (paged_page) before it addresses anything.
struct PagedBatch {
  const int32_t* q_start;      // [n_seqs + 1]
  const int32_t* kv_len;       // [n_seqs]
  const int32_t* page_table;   // [n_seqs][table_stride]
  int64_t table_stride;
  int32_t n_seqs;
  int32_t n_tokens;
  int32_t max_pages;           // columns of page_table
  int32_t num_pages;           // pages of the pool
  int32_t page_shift;          // log2 of the tokens per page
  int32_t kv_heads;
  int32_t group;               // query heads per kv head
  uint32_t group_magic;        // ceil(2^(31 + group_shift) / group)
  int32_t group_shift;         // ceil(log2(group))
  int32_t window;              // -1: no bound
  int32_t anchor_tokens;
  int32_t block;               // 1: the new tokens see each other
};

// Token of row r (r / group; exact for 0 <= r < 2^31: the magic number is off by less than
// group <= 2^group_shift in 2^(31 + group_shift)), a fifth of a division's instructions
__device__ inline int paged_token(const PagedBatch& b, int r) {
  return int(__umulhi(2u * uint32_t(r), b.group_magic) >> b.group_shift);
}

// Sequence s: its new tokens are rows q0 .. q0 + n_new - 1; token tau has index
// first + tau (negative: there is no such token); keys 0 .. keys - 1 are in its pages.
struct PagedSeq {
  int q0, n_new, first, keys;
};

__device__ inline PagedSeq paged_seq(const PagedBatch& b, int s) {
  PagedSeq q;
  q.q0 = min(max(b.q_start[s], 0), b.n_tokens);
  q.n_new = max(min(max(b.q_start[s + 1], 0), b.n_tokens) - q.q0, 0);
  const int len = max(b.kv_len[s], 0);
  q.first = len - q.n_new;
  q.keys = min(len, b.max_pages << b.page_shift);
  return q;
}

// Keys that token tau sees: j < hi and (j >= lo or j < anchor_tokens).
struct PagedRange {
  int lo, hi;
};

__device__ inline PagedRange paged_range(const PagedBatch& b, const PagedSeq& q, int tau) {
  const int i = b.block ? q.first : q.first + tau;
  PagedRange r;
  r.hi = b.block ? q.keys : min(q.keys, max(i + 1, 0));
  r.lo = b.window < 0 ? 0 : max(max(i, 0) - b.window, 0);
  return r;
}

// The blocks of KB keys that tokens tau0 .. tau1 read between them: n_anchor blocks from
// key 0, then those from block lo_block on; n in all.
template <int KB>
struct PagedBlocks {
  int n_anchor, lo_block, n;
  __device__ int key0(int t) const { return KB * (t < n_anchor ? t : lo_block + t - n_anchor); }
};

template <int KB>
__device__ inline PagedBlocks<KB> paged_blocks(const PagedBatch& b, const PagedRange& first,
                                               const PagedRange& last) {
  PagedBlocks<KB> p;
  p.lo_block = first.lo / KB;
  p.n_anchor = (min(min(b.anchor_tokens, first.lo), last.hi) + KB - 1) / KB;
  if (p.n_anchor >= p.lo_block) p.n_anchor = p.lo_block = 0;
  p.n = p.n_anchor + max((last.hi + KB - 1) / KB - p.lo_block, 0);
  return p;
}

// Work items.  A sequence's rows (row r: token r / group, query head r % group of the kv
// head) are cut into tiles of RT rows, the blocks that a tile reads into `parts` equal
// parts; an item is (sequence, tile, part), and every kv head runs all of them.  Lengths
// are known on the device only, so every wave finds its item by itself: it reads the
// batch's q_start and kv_len (one element per lane) and sums in lane order, the same in
// every wave.  Parts are of `per` blocks or a little less: `per` makes the whole batch, N
// tiles, max(target, spread * N) items or a little fewer, and is at least min_per.  So a
// ragged batch is divided by its total, not by its longest sequence, and a batch of no
// more tiles than that (spread 0 or 1) is not divided.  Sequences of min_rows < rows <=
// max_rows take part.
struct PagedSplit {
  int32_t target;     // 0: no parts
  int32_t spread;
  int32_t min_per;    // blocks
  int32_t min_rows, max_rows;
};

// Most tiles of n_seqs sequences of `rows` rows in all, and most items per kv head of a
// batch of at most `tiles` tiles.
inline int64_t paged_max_tiles(int64_t rows, int64_t n_seqs, int rt) {
  return (rows + (rt - 1) * n_seqs) / rt;
}

inline int64_t paged_max_items(int64_t tiles, const PagedSplit& sp) {
  if (sp.target == 0) return tiles;
  const int64_t most = sp.spread * tiles > sp.target ? sp.spread * tiles : sp.target;
  return most > tiles ? most : tiles;
}

// A value that every lane holds alike, in a scalar register
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ inline int64_t uniform(int64_t x) {
  const uint32_t lo = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uint64_t(x)))));
  const uint32_t hi = uint32_t(__builtin_amdgcn_readfirstlane(int(uint32_t(uint64_t(x) >> 32))));
  return int64_t((uint64_t(hi) << 32) | lo);
}

struct PagedItem {
  PagedSeq seq;
  int s, tile, part, parts;
  int item0;          // the tile's first item
};

template <int RT, int KB>
struct PagedScan {
  const PagedBatch& b;
  const PagedSplit& sp;
  const int lane;
  PagedSeq seq0;         // sequence `lane`
  int tiles0, blocks0;
  int per;               // blocks of a part, 0: no parts

  __device__ PagedScan(const PagedBatch& batch, const PagedSplit& split, int l)
      : b(batch), sp(split), lane(l), per(0) {
    of_sequence(lane, &seq0, &tiles0, &blocks0);
    if (sp.target > 0) per = blocks_per_part();
  }

  // sequence s, its tiles and an upper bound of the blocks of any of them, 0 tiles where s
  // takes no part
  __device__ void of_sequence(int s, PagedSeq* seq, int* tiles, int* blocks) const {
    *tiles = *blocks = 0;
    *seq = PagedSeq{0, 0, 0, 0};
    if (s >= b.n_seqs) return;
    const PagedSeq q = *seq = paged_seq(b, s);
    const int64_t rows = int64_t(q.n_new) * b.group;
    if (rows <= sp.min_rows || rows > sp.max_rows) return;
    *tiles = int((rows + RT - 1) / RT);
    int n = (q.keys + KB - 1) / KB;
    if (b.window >= 0) {
      const int64_t seen = int64_t(b.window) + b.anchor_tokens + (b.block ? q.n_new : RT) + 4 * KB;
      n = int(min(int64_t(n), seen / KB));
    }
    *blocks = n;
  }
  __device__ void of_lane(int s0, PagedSeq* seq, int* tiles, int* blocks) const {
    if (s0 == 0) {
      *seq = seq0;
      *tiles = tiles0;
      *blocks = blocks0;
    } else {
      of_sequence(s0 + lane, seq, tiles, blocks);
    }
  }
  __device__ int parts_of(int blocks) const { return per > 0 ? max((blocks + per - 1) / per, 1) : 1; }

  __device__ int blocks_per_part() const {
    float total = 0.0f, n = 0.0f;
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
      PagedSeq seq;
      int tiles, blocks;
      of_lane(s0, &seq, &tiles, &blocks);
      total += float(tiles) * float(blocks);
      n += float(tiles);
    }
    for (int d = 1; d < min(b.n_seqs, 64); d <<= 1) {   // (a lane behind the sequences has 0)
      total += __shfl_xor(total, d);
      n += __shfl_xor(n, d);
    }
    total = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(total)));
    n = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(n)));
    const float more = fmaxf(float(sp.target), float(sp.spread) * n) - n;   // items beyond one per tile
    if (more < 1.0f) return 1 << 30;
    // (the factor covers the rounding of the float32 sums: never more items than the bound)
    return max(sp.min_per, int(fminf(1.0001f * total / more, 1e9f)) + 1);
  }

  // Items of the batch
  __device__ int count() const {
    int all = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
      PagedSeq seq;
      int tiles, blocks;
      of_lane(s0, &seq, &tiles, &blocks);
      all += tiles * parts_of(blocks);
    }
    for (int d = 1; d < min(b.n_seqs, 64); d <<= 1) all += __shfl_xor(all, d);
    return uniform(all);
  }

  // The item `index`; false when the batch has fewer.  by_tile: index counts tiles, not
  // items (item0 and parts say which items a tile has).
  __device__ bool find(int index, bool by_tile, PagedItem* out) const {
    int before = 0, items_before = 0;   // of the sequences before s0
    for (int s0 = 0; s0 < b.n_seqs; s0 += 64) {
      PagedSeq seq;
      int tiles, blocks;
      of_lane(s0, &seq, &tiles, &blocks);
      const int parts = parts_of(blocks);
      const int items = tiles * parts;
      int sum = items, tsum = tiles;     // inclusive sums over the lanes
      for (int d = 1; d < min(b.n_seqs - s0, 64); d <<= 1) {
        const int a = __shfl_up(sum, d), t = __shfl_up(tsum, d);
        if (lane >= d) {
          sum += a;
          tsum += t;
        }
      }
      const int rel = index - before;
      const uint64_t hit = __builtin_amdgcn_ballot_w64((by_tile ? tsum : sum) > rel);
      if (hit != 0) {
        const int l = __builtin_ctzll(hit);
        const int n_parts = __builtin_amdgcn_readlane(parts, l);
        const int n_tiles = __builtin_amdgcn_readlane(tiles, l);
        const int sum_l = __builtin_amdgcn_readlane(sum, l), tsum_l = __builtin_amdgcn_readlane(tsum, l);
        const int in_seq = rel - (by_tile ? tsum_l - n_tiles : sum_l - n_tiles * n_parts);
        // (every lane holds the same: kept where the addresses made of it stay scalar)
        const int tile = by_tile ? in_seq : in_seq / n_parts;
        out->s = uniform(s0 + l);
        out->seq = {__builtin_amdgcn_readlane(seq.q0, l), __builtin_amdgcn_readlane(seq.n_new, l),
                    __builtin_amdgcn_readlane(seq.first, l), __builtin_amdgcn_readlane(seq.keys, l)};
        out->parts = uniform(n_parts);
        out->tile = uniform(tile);
        out->part = uniform(by_tile ? 0 : in_seq - tile * n_parts);
        out->item0 = uniform(items_before + sum_l - n_tiles * n_parts + tile * n_parts);
        // (sums that ran over, which only a broken q_start can cause, name no item)
        return in_seq >= 0 && out->tile < n_tiles && out->item0 >= 0;
      }
      // (only a block of 64 sequences has another behind it)
      const int all = __builtin_amdgcn_readlane(sum, 63);
      before += by_tile ? __builtin_amdgcn_readlane(tsum, 63) : all;
      items_before += all;
    }
    return false;
  }
};

// The page that holds key j of sequence s, -1 for a hole (a table entry that names no
// page of the pool, or a key behind the table).
__device__ inline int paged_page(const PagedBatch& b, int s, int j) {
  const int col = j >> b.page_shift;
  if (j < 0 || col >= b.max_pages) return -1;
  const int p = b.page_table[int64_t(s) * b.table_stride + col];
  return uint32_t(p) < uint32_t(b.num_pages) ? p : -1;
}

}  // namespace ff
