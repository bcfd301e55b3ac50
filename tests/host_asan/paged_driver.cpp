// Drives the paged cache's entry points (include/ff_paged.h) with host-only stand-ins for
// its launches, under AddressSanitizer and UndefinedBehaviorSanitizer: what a launch gets
// must lie within what the call was given.  Test infrastructure only.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "ff_paged.h"
#include "ff_paged_internal.h"

static int launches = 0;
static size_t workspace_used = 0;
static void* const device = reinterpret_cast<void*>(uintptr_t(0x7f0000000000));

namespace ff {

static hipError_t batch_ok(const PagedBatch& b) {
  const bool ok = b.n_seqs >= 1 && b.n_tokens >= 1 && b.max_pages >= 1 && b.page_shift >= 4 &&
                  b.page_shift <= 8 && b.group >= 1 && b.kv_heads >= 1 && b.window >= -1 &&
                  b.q_start && b.kv_len && b.page_table && b.table_stride >= b.max_pages;
  ++launches;
  return ok ? hipSuccess : hipErrorInvalidValue;
}

// items: at least as many as the launch's sequences can have tiles, or the target
static hipError_t attention_ok(int rows, const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                               int64_t items, int head_dim) {
  const int64_t all = int64_t(b.n_tokens) * b.group;
  int64_t tiles = all / rows;                                    // one sequence has them all
  if (sp.max_rows < INT32_MAX)                                   // or every sequence its most
    tiles = std::min(all / sp.max_rows, int64_t(b.n_seqs)) * ((sp.max_rows + rows - 1) / rows);
  if (items < tiles || items < sp.target) return hipErrorInvalidValue;
  if (sp.target > 0) {
    if (!t.part || reinterpret_cast<uintptr_t>(t.part) % 16 != 0) return hipErrorInvalidValue;
    const char* end = reinterpret_cast<const char*>(t.part) + size_t(items) * b.kv_heads * paged_part_floats(rows, head_dim) * 4;
    workspace_used = std::max(workspace_used, size_t(end - static_cast<const char*>(device)));
  }
  return batch_ok(b);
}

hipError_t launch_paged_append(const PagedBatch& b, const PagedAppend& a, int head_dim, int, hipStream_t) {
  for (int p = 0; p < head_dim / 2; ++p)
    if (!(a.omega[p] > 0.0)) return hipErrorInvalidValue;
  return batch_ok(b);
}
hipError_t launch_paged_attn_bf16(int qt, int, bool, const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                                  int64_t items, int head_dim, hipStream_t) {
  return attention_ok(16 * qt, b, sp, t, items, head_dim);
}
hipError_t launch_paged_attn_f32(int qt, bool, const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t,
                                 int64_t items, int head_dim, hipStream_t) {
  return attention_ok(16 * qt, b, sp, t, items, head_dim);
}
hipError_t launch_paged_prompt(const PagedBatch& b, const PagedSplit& sp, const PagedTensors& t, int64_t items,
                               int head_dim, hipStream_t) {
  return attention_ok(kPagedPromptRows, b, sp, t, items, head_dim);
}
hipError_t launch_paged_join(int, int, const PagedBatch& b, const PagedSplit& sp, const PagedTensors&, int64_t,
                             int64_t, int, int, hipStream_t) {
  return sp.target > 0 ? batch_ok(b) : hipErrorInvalidValue;
}

}  // namespace ff

#define CHECK(x)                                                            \
  do {                                                                      \
    if (!(x)) {                                                             \
      std::printf("line %d: %s (%s)\n", __LINE__, #x, ff_last_error());     \
      std::exit(1);                                                         \
    }                                                                       \
  } while (0)

int main() {
  void* dev = device;
  const int32_t* ints = static_cast<const int32_t*>(dev);
  ff_paged_rope rope = {0, 0, 0, 0, 10000.0};
  int calls = 0;
  for (int dtype = 0; dtype < 2; ++dtype)
    for (int d : {64, 128})
      for (int page : {16, 64, 256})
        for (int kv : {1, 3, 8})
          for (int group : {1, 5, 16})
            for (int seqs : {0, 1, 70, 1024})
              for (int tokens : {0, 1, 257, 100000})
                for (int pages : {1, 40, 4000000})
                  for (int max_new : {0, 1, INT_MAX}) {
                    ff_paged_desc p;
                    std::memset(&p, 0, sizeof(p));
                    p.num_pages = INT_MAX;
                    p.page_tokens = page;
                    p.num_q_heads = kv * group;
                    p.num_kv_heads = kv;
                    p.head_dim = d;
                    p.dtype = dtype;
                    p.n_seqs = seqs;
                    p.n_tokens = tokens;
                    p.max_pages = pages;
                    p.max_new = max_new;
                    p.table_stride = pages + 3;
                    p.q_start = p.kv_len = p.page_table = ints;
                    const int64_t stride = int64_t(kv) * group * d + 64;
                    const size_t need = ff_paged_attention_workspace(&p);
                    workspace_used = 0;
                    ff_status st = ff_paged_attention(&p, dev, stride, dev, dev, dev, nullptr, 0.1f, 0, INT_MAX,
                                                      INT_MAX, need ? dev : nullptr, need, nullptr);
                    CHECK(st == (int64_t(pages) * page > (1 << 30) ? FF_ERR_UNSUPPORTED : FF_OK) || st == FF_ERR_UNSUPPORTED);
                    CHECK(workspace_used <= need);
                    if (st == FF_OK && need > 0 && seqs > 0 && tokens > 0)
                      CHECK(ff_paged_attention(&p, dev, stride, dev, dev, dev, nullptr, 0.1f, 1, -1, 0, dev, need - 1,
                                               nullptr) == FF_ERR_BUFFER);
                    if (st == FF_OK)
                      CHECK(ff_paged_append(&p, &rope, dev, dev, dev, stride, stride, stride, nullptr,
                                            static_cast<char*>(dev) + 4096, dev, dev, nullptr) == FF_OK);
                    ++calls;
                  }
  CHECK(ff_paged_attention_workspace(nullptr) == 0);
  CHECK(ff_paged_append(nullptr, &rope, dev, dev, dev, 0, 0, 0, nullptr, dev, dev, dev, nullptr) == FF_ERR_INVALID_ARG);
  std::printf("paged host checks passed: %d calls, %d launches\n", calls, launches);
  return 0;
}
