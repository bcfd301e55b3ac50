// Host side of the paged cache: validation, launch choices and the C ABI entry points
// declared in include/ff_paged.h.  Stateless: lengths and pages stay on the device.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

#include "ff_paged.h"
#include "ff_paged_internal.h"

namespace {

using ff::fail;
using ff::ok;

ff_status check_aligned(const void* p, size_t to, const char* name) {
  if (reinterpret_cast<uintptr_t>(p) % to != 0)
    return fail(FF_ERR_INVALID_ARG, "%s must be %zu-byte aligned", name, to);
  return FF_OK;
}

ff_status hip_status(hipError_t e, const char* what) {
  if (e != hipSuccess) return fail(FF_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return ok();
}

int elem_bytes(const ff_paged_desc& d) { return d.dtype == FF_DT_BF16 ? 2 : 4; }

ff_status check_desc(const ff_paged_desc* d) {
  if (!d) return fail(FF_ERR_INVALID_ARG, "desc is NULL");
  if (d->num_pages < 1) return fail(FF_ERR_INVALID_ARG, "num_pages must be >= 1");
  if (d->page_tokens < FF_MIN_PAGE_TOKENS || d->page_tokens > FF_MAX_PAGE_TOKENS ||
      (d->page_tokens & (d->page_tokens - 1)) != 0)
    return fail(FF_ERR_UNSUPPORTED, "page_tokens must be a power of two in [%d, %d]",
                FF_MIN_PAGE_TOKENS, FF_MAX_PAGE_TOKENS);
  if (d->num_kv_heads < 1 || d->num_q_heads < 1)
    return fail(FF_ERR_INVALID_ARG, "num_kv_heads and num_q_heads must be >= 1");
  if (d->num_q_heads % d->num_kv_heads != 0)
    return fail(FF_ERR_SHAPE, "num_q_heads must be a multiple of num_kv_heads");
  if (d->head_dim != 64 && d->head_dim != 128)
    return fail(FF_ERR_UNSUPPORTED, "head_dim must be 64 or 128");
  if (d->dtype != FF_DT_BF16 && d->dtype != FF_DT_F32)
    return fail(FF_ERR_UNSUPPORTED, "dtype must be FF_DT_BF16 or FF_DT_F32");
  if (d->n_seqs < 0 || d->n_seqs > FF_MAX_PAGED_SEQS)
    return fail(FF_ERR_UNSUPPORTED, "n_seqs must be in [0, %d]", FF_MAX_PAGED_SEQS);
  if (d->n_tokens < 0) return fail(FF_ERR_INVALID_ARG, "n_tokens must be >= 0");
  if (d->min_new < 0 || d->max_new < 0 || (d->max_new > 0 && d->min_new > d->max_new))
    return fail(FF_ERR_INVALID_ARG, "min_new and max_new must be 0 <= min_new <= max_new");
  if (d->max_pages < 1) return fail(FF_ERR_INVALID_ARG, "max_pages must be >= 1");
  if (int64_t(d->max_pages) * d->page_tokens > (int64_t(1) << 30))
    return fail(FF_ERR_UNSUPPORTED, "max_pages * page_tokens must be at most 2^30");
  if (d->table_stride < d->max_pages)
    return fail(FF_ERR_SHAPE, "table_stride must be at least max_pages");
  // rows of a sequence and elements of a row of heads are counted in 32 bits
  if (int64_t(d->n_tokens) * (d->num_q_heads / d->num_kv_heads) > INT32_MAX - 256)
    return fail(FF_ERR_UNSUPPORTED, "n_tokens * query heads per kv head must fit in 32 bits");
  if (int64_t(d->num_q_heads) * d->head_dim > (1 << 24))
    return fail(FF_ERR_UNSUPPORTED, "num_q_heads * head_dim must be at most 2^24");
  if (d->n_seqs > 0) {
    if (!d->q_start || !d->kv_len || !d->page_table)
      return fail(FF_ERR_INVALID_ARG, "q_start, kv_len and page_table must be non-NULL");
    if (check_aligned(d->q_start, 4, "q_start") != FF_OK ||
        check_aligned(d->kv_len, 4, "kv_len") != FF_OK ||
        check_aligned(d->page_table, 4, "page_table") != FF_OK)
      return FF_ERR_INVALID_ARG;
  }
  return FF_OK;
}

// Rows of heads that are `stride` elements apart
ff_status check_rows(const ff_paged_desc& d, const void* p, int64_t stride, int heads,
                     const char* name) {
  if (!p) return fail(FF_ERR_INVALID_ARG, "%s is NULL", name);
  if (check_aligned(p, 16, name) != FF_OK) return FF_ERR_INVALID_ARG;
  if (stride < int64_t(heads) * d.head_dim || stride * elem_bytes(d) % 16 != 0 ||
      stride > (int64_t(1) << 31))
    return fail(FF_ERR_SHAPE, "the rows of %s must be a multiple of 16 bytes and at least "
                "%d heads of %d elements apart", name, heads, d.head_dim);
  return FF_OK;
}

ff::PagedBatch make_batch(const ff_paged_desc& d) {
  ff::PagedBatch b;
  std::memset(&b, 0, sizeof(b));
  b.q_start = d.q_start;
  b.kv_len = d.kv_len;
  b.page_table = d.page_table;
  b.table_stride = d.table_stride;
  b.n_seqs = d.n_seqs;
  b.n_tokens = d.n_tokens;
  b.max_pages = d.max_pages;
  b.num_pages = d.num_pages;
  b.page_shift = __builtin_ctz(unsigned(d.page_tokens));
  b.kv_heads = d.num_kv_heads;
  b.group = d.num_q_heads / d.num_kv_heads;
  while ((1 << b.group_shift) < b.group) ++b.group_shift;
  b.group_magic = uint32_t(((uint64_t(1) << (31 + b.group_shift)) + b.group - 1) / b.group);
  b.window = -1;
  return b;
}

// Launch choices of one attention call: they follow from sizes, so that the workspace can
// be asked for ahead of it.
struct Launch {
  int rows;              // of a tile: 16, 32 or kPagedPromptRows; 0: no launch
  int used;              // of them, where the batch is as its hints say
  ff::PagedSplit split;
  int64_t tiles, items;  // at most this many per kv head
  size_t part_bytes;     // of its partial results
  int waves;             // few rows: waves of a workgroup
  bool once;             // and whether every sequence is one tile
};
struct Plan {
  Launch few, many;      // sequences of few rows, and of many
};

// Rows (new tokens x query heads per kv head) above which a sequence goes to the kernel of
// 256-row tiles where a batch runs both: up to here one tile of the other reads each key
// once.
constexpr int kManyRows = 32;

// Whether a bf16 batch runs on the kernel of few rows alone, by estimated times (us).  That
// kernel reads the keys once from HBM, and again, mostly from L2, for every further tile of
// 32 rows.  The other takes equal time for its key blocks, but one tile's at the least, and a
// fixed part for prologue, partials and join, and for the first one's launch where that is
// needed as well.  The constants are fits to 1 to 64 sequences x 48 to 256 rows x 300 to 30000
// keys and to prompts of 20 to 2000 tokens, either kernel forced: 2 sequences x 588 tokens over
// 2350 keys, 2 heads 24 against 34; 5 prompts of up to 300 tokens, 5 heads 11 against 31; 8 x 48
// rows x 4000 keys, 12 heads 80 against 55; 1170 tokens over 7000 keys, 12 heads 132 against 69.
// Keys are counted by the table's columns.
bool few_rows_alone(const ff_paged_desc& d, int64_t rows, bool both, double keys, int cus) {
  const double seqs = std::min(d.n_seqs, d.n_tokens);
  const double key_bytes = 4.0 * d.head_dim * d.num_kv_heads;
  const double more = std::max(double(rows) / 32 - 0.5 * seqs, 0.0);   // tiles beyond one each
  const double few = 8.0 + seqs * keys * key_bytes / 5.5e6 + more * keys * key_bytes / 9e6;
  const double step = d.head_dim == 128 ? 1.7 : 1.0;   // a 64-key block of a 256-row tile
  const double units = double(ff::paged_max_tiles(rows, int64_t(seqs), ff::kPagedPromptRows)) * d.num_kv_heads;
  const double many = 20.0 + (both ? 10.0 : 0.0) + step * std::max(units * keys / 64 / cus, std::min(keys / 64, 8.0));
  return few <= many;
}

// Parts of each of `tiles` float32 tiles of 32 rows of long prompts, which the matrix unit
// bounds: a CU runs a whole number of parts, every part adds 5 us, and the join 6 and the
// partials' way to HBM and back (5 TB/s).  Against as many parts as make two items per CU: 188
// tiles over 4500 keys 186 us and 150 (4 parts each instead of 2), 207 over 8700 339 and 303.
// The keys are cut for a gain of 3% and more, which many rounds of tiles do not leave, and into
// at most 16 items per CU, so that the workspace stays within 70 MB (256 CUs).
int parts_of_f32_tiles(const ff_paged_desc& d, int64_t tiles, double keys, int cus) {
  const double tile = keys / 64 * (d.head_dim == 128 ? 2.4 : 1.3);   // us on one CU
  const double moved = double(tiles) * ff::paged_part_floats(32, d.head_dim) * 4 * 2 / 5e6;   // us per part
  int best = 1;
  double least = 0.97 * double((tiles + cus - 1) / cus) * (tile + 5.0);
  // (p + 1 parts of a tile bound the items of a ragged batch)
  for (int p = 2; p <= 16 && tiles * (p + 1) <= 16 * cus; ++p) {
    const double us = double((tiles * p + cus - 1) / cus) * (tile / p + 5.0) + 6.0 + p * moved;
    if (us < least) {
      best = p;
      least = us;
    }
  }
  return best;
}

// blocks: of the longest sequence; none is cut that has no more than `whole` of them
void set_items(const ff_paged_desc& d, Launch* l, int64_t blocks, int64_t whole) {
  if (blocks <= whole) l->split.target = 0;
  l->items = ff::paged_max_items(l->tiles, l->split);
  l->part_bytes = l->split.target > 0 ? size_t(l->items) * d.num_kv_heads *
                                            ff::paged_part_floats(l->rows, d.head_dim) * 4 : 0;
}

Plan make_plan(const ff_paged_desc& d) {
  Plan p;
  std::memset(&p, 0, sizeof(p));
  const int group = d.num_q_heads / d.num_kv_heads, cus = ff::device_cus();
  const int64_t rows = int64_t(d.n_tokens) * group;
  const int64_t most = (d.max_new > 0 ? std::min(d.max_new, d.n_tokens) : d.n_tokens) * int64_t(group);
  const int64_t keys = int64_t(d.max_pages) * d.page_tokens;
  const bool bf16 = d.dtype == FF_DT_BF16;
  const bool some_few = int64_t(d.min_new) * group <= kManyRows;
  const bool many = bf16 && most > kManyRows && !few_rows_alone(d, rows, some_few, double(keys), cus);
  const bool few = !many || some_few;
  if (few) {
    Launch& l = p.few;
    l.rows = most <= 16 ? 16 : 32;
    l.used = int(std::min(most, int64_t(l.rows)));
    l.split.min_rows = 0;
    l.split.max_rows = many ? kManyRows : INT32_MAX;
    l.tiles = ff::paged_max_tiles(rows, d.n_seqs, l.rows);
    if (many) l.tiles = std::min(l.tiles, int64_t(d.n_seqs) * ((kManyRows + l.rows - 1) / l.rows));
    const int block = bf16 ? 32 : 16;
    l.split.min_per = 256 / block;
    l.split.target = (2 * cus + d.num_kv_heads - 1) / d.num_kv_heads;
    l.split.spread = l.tiles * d.num_kv_heads <= 16 * cus ? (bf16 ? 4 : 2) : 0;
    // (fewer tiles per sequence are bound by the keys' bytes: 10 sequences of 48 rows over up to
    // 23000 keys 93 us by this rule, 54 without)
    if (!bf16 && rows >= 4 * int64_t(l.rows) * d.n_seqs) {
      const int parts = parts_of_f32_tiles(d, l.tiles * d.num_kv_heads, double(keys), cus);
      l.split.target = parts > 1 ? 1 : 0;
      l.split.spread = parts + 1;
    }
    set_items(d, &l, (keys + block - 1) / block, 1024 / block);
    // Short caches in more workgroups than two per CU: two waves each (no more of their
    // blocks than two waves' copies cover are left for four), twice as many sequences at once.
    l.waves = bf16 && keys <= 512 && l.tiles * d.num_kv_heads > 2 * cus ? 2 : 4;
    l.once = most <= l.rows;
  }
  if (many) {
    Launch& l = p.many;
    l.rows = l.used = ff::kPagedPromptRows;
    l.split.min_rows = few ? kManyRows : 0;
    l.split.max_rows = INT32_MAX;
    l.tiles = ff::paged_max_tiles(rows, few ? std::min(int64_t(d.n_seqs), rows / kManyRows) : d.n_seqs, l.rows);
    l.split.min_per = 8;
    // Parts for launches of fewer tiles than CUs.  From three quarters of them on there is
    // nothing to gain (two prompts of 5000 and 4000 tokens, 32/8 heads: 361 us with the join
    // that finds no parts, 355 without), and parts that even out tiles of unequal length cost
    // more in partials than they save (spread 2 to 4 for a mixed batch: 142 us to 154 to 180).
    l.split.target = 4 * l.tiles * d.num_kv_heads >= 3 * cus ? 0 : std::max(cus / d.num_kv_heads, 1);
    l.split.spread = 0;
    set_items(d, &l, (keys + 63) / 64, l.split.min_per);
  }
  return p;
}

// The forms that the calling thread's last attention call took (exported as
// ff_internal_last_paged, not part of the C ABI), so that a test can tell that it reached
// the one it is about: rows of a tile of few rows (0: not launched) and whether its keys
// could be cut, the same of many rows; of few rows also the waves of a workgroup and
// whether the keys are read past the caches.
thread_local int32_t last_paged[6] = {};

hipError_t run(const Launch& l, const ff_paged_desc& d, const ff::PagedBatch& b,
               const ff::PagedTensors& t, hipStream_t stream) {
  hipError_t e;
  if (l.rows == ff::kPagedPromptRows)
    e = ff::launch_paged_prompt(b, l.split, t, l.items, d.head_dim, stream);
  else if (d.dtype == FF_DT_BF16)
    e = ff::launch_paged_attn_bf16(l.rows / 16, l.waves, l.once, b, l.split, t, l.items, d.head_dim, stream);
  else
    e = ff::launch_paged_attn_f32(l.rows / 16, l.once, b, l.split, t, l.items, d.head_dim, stream);
  if (e == hipSuccess && l.split.target > 0)
    e = ff::launch_paged_join(l.rows, l.used, b, l.split, t, l.items, l.tiles, d.head_dim, d.dtype, stream);
  return e;
}

}  // namespace

extern "C" {

int32_t ff_internal_last_paged(int32_t field) { return field >= 0 && field < 6 ? last_paged[field] : -1; }

ff_status ff_paged_append(const ff_paged_desc* desc, const ff_paged_rope* rope, const void* q,
                          const void* k, const void* v, int64_t q_stride, int64_t k_stride,
                          int64_t v_stride, const int32_t* positions, void* q_out, void* k_pages,
                          void* v_pages, void* stream) {
  ff_status st = check_desc(desc);
  if (st != FF_OK) return st;
  const ff_paged_desc& d = *desc;
  if (!rope) return fail(FF_ERR_INVALID_ARG, "rope is NULL");
  ff_paged_rope r = *rope;
  ff::resolve_rope_pairs(d.head_dim, &r.rope_pairs_t, &r.rope_pairs_h, &r.rope_pairs_w);
  const int64_t pairs = int64_t(r.rope_pairs_t) + r.rope_pairs_h + r.rope_pairs_w;
  if (r.rope_pairs_t < 0 || r.rope_pairs_h < 0 || r.rope_pairs_w < 0 || pairs != d.head_dim / 2)
    return fail(FF_ERR_INVALID_ARG, "rope pairs must be >= 0 and sum to head_dim / 2");
  if (!(r.rope_theta > 0.0) || !std::isfinite(r.rope_theta))
    return fail(FF_ERR_INVALID_ARG, "rope_theta must be positive");
  if (d.n_seqs == 0 || d.n_tokens == 0) return ok();
  // (a grid holds at most 2^32 - 1 threads)
  if (d.n_tokens > int64_t(UINT32_MAX) / 256)
    return fail(FF_ERR_UNSUPPORTED, "too many rows for one launch");
  if ((st = check_rows(d, k, k_stride, d.num_kv_heads, "k")) != FF_OK) return st;
  if ((st = check_rows(d, v, v_stride, d.num_kv_heads, "v")) != FF_OK) return st;
  if (q) {
    if ((st = check_rows(d, q, q_stride, d.num_q_heads, "q")) != FF_OK) return st;
    if (!q_out) return fail(FF_ERR_INVALID_ARG, "q_out is NULL");
    if (check_aligned(q_out, 16, "q_out") != FF_OK) return FF_ERR_INVALID_ARG;
    if (q_out == q && q_stride != int64_t(d.num_q_heads) * d.head_dim)
      return fail(FF_ERR_SHAPE, "q_out may be q only when q is dense");
  }
  if (!k_pages || !v_pages) return fail(FF_ERR_INVALID_ARG, "k_pages and v_pages must be non-NULL");
  if (check_aligned(k_pages, 16, "k_pages") != FF_OK || check_aligned(v_pages, 16, "v_pages") != FF_OK ||
      check_aligned(positions, 4, "positions") != FF_OK)
    return FF_ERR_INVALID_ARG;
  ff::PagedAppend a;
  std::memset(&a, 0, sizeof(a));
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.positions = positions;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.n_t = r.rope_pairs_t;
  a.n_th = r.rope_pairs_t + r.rope_pairs_h;
  ff::rope_frequencies(r.rope_pairs_t, r.rope_pairs_h, r.rope_pairs_w, r.rope_theta, a.omega);
  return hip_status(ff::launch_paged_append(make_batch(d), a, d.head_dim, d.dtype,
                                            static_cast<hipStream_t>(stream)),
                    "paged_append launch");
}

size_t ff_paged_attention_workspace(const ff_paged_desc* desc) {
  if (check_desc(desc) != FF_OK) return 0;
  ok();
  const Plan p = make_plan(*desc);
  return p.few.part_bytes + p.many.part_bytes;
}

ff_status ff_paged_attention(const ff_paged_desc* desc, const void* q, int64_t q_stride,
                             const void* k_pages, const void* v_pages, void* out, float* lse,
                             float softmax_scale, int32_t block, int32_t window,
                             int32_t anchor_tokens, void* workspace, size_t workspace_bytes,
                             void* stream) {
  ff_status st = check_desc(desc);
  if (st != FF_OK) return st;
  const ff_paged_desc& d = *desc;
  if (!(softmax_scale > 0.0f) || !std::isfinite(softmax_scale))
    return fail(FF_ERR_INVALID_ARG, "softmax_scale must be positive and finite");
  if (block != 0 && block != 1) return fail(FF_ERR_INVALID_ARG, "block must be 0 or 1");
  if (window < -1) return fail(FF_ERR_INVALID_ARG, "window must be -1 or >= 0");
  if (anchor_tokens < 0) return fail(FF_ERR_INVALID_ARG, "anchor_tokens must be >= 0");
  if (d.n_seqs == 0 || d.n_tokens == 0) return ok();
  if ((st = check_rows(d, q, q_stride, d.num_q_heads, "q")) != FF_OK) return st;
  if (!k_pages || !v_pages || !out)
    return fail(FF_ERR_INVALID_ARG, "k_pages, v_pages and out must be non-NULL");
  if (check_aligned(k_pages, 16, "k_pages") != FF_OK || check_aligned(v_pages, 16, "v_pages") != FF_OK ||
      check_aligned(out, 16, "out") != FF_OK || check_aligned(lse, 4, "lse") != FF_OK ||
      check_aligned(workspace, 16, "workspace") != FF_OK)
    return FF_ERR_INVALID_ARG;
  const Plan p = make_plan(d);
  const size_t need = p.few.part_bytes + p.many.part_bytes;
  if (need > 0 && !workspace) return fail(FF_ERR_INVALID_ARG, "workspace is NULL");
  if (workspace_bytes < need)
    return fail(FF_ERR_BUFFER, "workspace_bytes %zu < required %zu", workspace_bytes, need);
  // (a grid holds at most 2^32 - 1 threads)
  if (std::max(p.few.items, p.many.items) * d.num_kv_heads > int64_t(UINT32_MAX) / 512)
    return fail(FF_ERR_UNSUPPORTED, "too many rows for one launch");
  ff::PagedBatch b = make_batch(d);
  b.window = std::min(window, 1 << 30);
  b.anchor_tokens = std::min(anchor_tokens, 1 << 30);
  b.block = block;
  ff::PagedTensors t;
  std::memset(&t, 0, sizeof(t));
  t.q = q;
  t.out = out;
  t.lse = lse;
  t.k_pages = k_pages;
  t.v_pages = v_pages;
  t.part = static_cast<float*>(workspace);
  t.q_stride = q_stride;
  t.scale = softmax_scale;
  t.scale_log2 = float(double(softmax_scale) * 1.4426950408889634);
  const hipStream_t hs = static_cast<hipStream_t>(stream);
  const int32_t forms[6] = {p.few.rows, p.few.split.target > 0, p.many.rows, p.many.split.target > 0,
                            p.few.waves, p.few.once};
  std::copy(forms, forms + 6, last_paged);
  hipError_t e = hipSuccess;
  if (p.few.rows > 0) e = run(p.few, d, b, t, hs);
  t.part = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.few.part_bytes);
  if (e == hipSuccess && p.many.rows > 0) e = run(p.many, d, b, t, hs);
  return hip_status(e, "paged_attention launch");
}

}  // extern "C"
