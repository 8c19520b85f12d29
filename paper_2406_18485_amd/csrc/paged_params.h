// Arguments of the paged attention kernels, and how a launch of either is sized.
#pragma once
#include <stdint.h>

#include "loong_internal.h"

namespace loong {

constexpr int kWin = 1024;             // pages whose places are in LDS
constexpr int kFewRows = 32;           // query rows of a kv head up to which the kernel for few is taken

struct PagedParams {
  const uint16_t *q, *k, *v;
  const int32_t *seq_start, *kv_len, *table;
  float *out, *lse;
  uint16_t* o;
  int64_t qs[2], os[2], cs[3], ts;
  int32_t n_seqs, n_tokens, max_new, hq, hkv, G;
  int32_t n_pages, max_pages, page_size;
  int32_t cap;          // keys that a row of the page table has pages for
  uint32_t page_mul;    // key / page_size = mulhi(2 key, page_mul) >> page_shift
  int32_t page_shift;
  float c;              // softmax_scale * log2(e)
  int32_t causal;
  uint32_t* counters;
  float* parts;
  int32_t slot_floats;
};

// Workgroups of a launch, and the partial results that it may have at a time.
struct PagedPlan {
  int64_t workgroups, slots;
  int slot_floats;
};
// keys that a sequence has pages for (2^30 at the most)
inline int64_t cached_keys(const loong_paged_desc& d) { return (int64_t)d.max_pages * d.page_size; }
PagedPlan plan_paged_few(const loong_paged_desc& d, int cus);
PagedPlan plan_paged_many(const loong_paged_desc& d, int cus);
void launch_paged_few(const PagedParams& p, const loong_paged_desc& d, unsigned grid, void* stream);
void launch_paged_many(const PagedParams& p, const loong_paged_desc& d, int cus, unsigned grid, void* stream);

}  // namespace loong
