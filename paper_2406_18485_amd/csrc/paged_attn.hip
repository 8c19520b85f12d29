// Attention of new tokens over a paged cache: arguments, and which kernel.
//
// Rows.  The query rows of one kv head (new tokens x the group's q heads, token by token) are stacked, so that all of them share
// the keys that are read for them; a row's last visible key follows from its token.  As in the forward step, S^T = K Q^T puts a
// query row into one lane (softmax statistics in the lane, one exchange with the lane 32 places away) and the probabilities into
// the operand layout of O^T += V^T P^T.  Few rows a kv head (paged_few.hip) are bound by HBM, many (paged_many.hip) by the matrix cores.
//
// Lengths are in device memory, so a launch is made for what they may be at most, and the kernels work out the division of the work
// from what they are.
//
// Pages.  The page numbers that a workgroup needs lie in LDS (`win`), checked once: a number outside the cache becomes page 0,
// and rows that would see its keys are NaN at the end.  A lane finds the address of the piece that it stages from there.
#include <hip/hip_runtime.h>

#include <cmath>

#include "paged_params.h"

namespace loong {
namespace {

// few rows of a kv head in every sequence?
bool is_few(const loong_paged_desc& d) {
  const int64_t most = d.max_new < d.n_tokens ? d.max_new : d.n_tokens;
  return most * (d.n_q_heads / d.n_kv_heads) <= kFewRows;
}
PagedPlan plan_paged(const loong_paged_desc& d, int cus) { return is_few(d) ? plan_paged_few(d, cus) : plan_paged_many(d, cus); }
int64_t workspace_of(const PagedPlan& pl) { return pl.slots ? kWsHeadBytes + pl.slots * pl.slot_floats * 4 : 0; }

int check_attn(const loong_paged_desc* d) {
  if (int rc = check_paged(d, LOONG_WORKSPACE_CLEAN)) return rc;
  if (!std::isfinite(d->softmax_scale) || d->softmax_scale <= 0.f) return fail(LOONG_E_SHAPE, "softmax_scale must be finite and positive");
  return LOONG_OK;
}

}  // namespace
}  // namespace loong

using namespace loong;

extern "C" {

int loong_paged_workspace_bytes(const loong_paged_desc* desc, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(LOONG_E_NULL, "loong_paged_workspace_bytes: NULL result");
  if (int rc = check_attn(desc)) return rc;
  *bytes = workspace_of(plan_paged(*desc, planning_cus()));
  return LOONG_OK;
}

int loong_paged_attn(const loong_paged_desc* desc, const void* q, const void* k_cache, const void* v_cache, const int32_t* seq_start,
                     const int32_t* kv_len, const int32_t* page_table, float* out, void* o, float* lse, void* workspace,
                     int64_t workspace_bytes, void* stream) {
  clear_error();
  if (int rc = check_attn(desc)) return rc;
  const loong_paged_desc& d = *desc;
  if (!q || !k_cache || !v_cache || !seq_start || !kv_len || !page_table || !lse || (!out && !o)) return fail(LOONG_E_NULL, "loong_paged_attn: NULL argument");
  for (const void* x : {q, k_cache, v_cache, (const void*)out, (const void*)o, (const void*)workspace})
    if (!aligned16(x)) return fail(LOONG_E_ALIGN, "loong_paged_attn: tensor not 16-byte aligned");
  for (const void* x : {(const void*)seq_start, (const void*)kv_len, (const void*)page_table, (const void*)lse})
    if (reinterpret_cast<uintptr_t>(x) & 3) return fail(LOONG_E_ALIGN, "loong_paged_attn: table or lse not 4-byte aligned");
  if (d.n_tokens == 0 || d.n_seqs == 0 || d.max_new == 0) return LOONG_OK;
  const int64_t rows[2] = {d.n_tokens, d.n_q_heads};
  for (int i = 0; i < 2; ++i)
    if (!apart(d.o_stride[i], rows[i], d.head_dim)) return fail(LOONG_E_SHAPE, "o_stride[%d] = %lld: rows of a result lie on each other", i, (long long)d.o_stride[i]);
  if (d.n_pages == 0) return fail(LOONG_E_SHAPE, "loong_paged_attn: a cache without pages");
  DeviceFacts dev;
  if (int rc = device_facts(&dev)) return rc;
  const PagedPlan pl = plan_paged(d, dev.cus);
  const int64_t need = workspace_of(pl);
  if (need > 0) {
    if (!workspace) return fail(LOONG_E_NULL, "loong_paged_attn: NULL workspace");
    if (workspace_bytes < need)
      return fail(LOONG_E_SHAPE, "loong_paged_attn: workspace of %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
  }
  if (!launch_fits(pl.workgroups, 512)) return fail(LOONG_E_UNSUPPORTED, "loong_paged_attn: grid too large");
  PagedParams p{};
  p.q = (const uint16_t*)q; p.k = (const uint16_t*)k_cache; p.v = (const uint16_t*)v_cache;
  p.seq_start = seq_start; p.kv_len = kv_len; p.table = page_table;
  p.out = out; p.lse = lse; p.o = (uint16_t*)o;
  for (int i = 0; i < 2; ++i) { p.qs[i] = d.q_stride[i]; p.os[i] = d.o_stride[i]; }
  for (int i = 0; i < 3; ++i) p.cs[i] = d.cache_stride[i];
  p.ts = d.table_stride;
  p.n_seqs = d.n_seqs; p.n_tokens = d.n_tokens; p.max_new = d.max_new; p.hq = d.n_q_heads; p.hkv = d.n_kv_heads; p.G = d.n_q_heads / d.n_kv_heads;
  p.n_pages = d.n_pages; p.max_pages = d.max_pages; p.page_size = d.page_size;
  p.cap = (int32_t)cached_keys(d);
  // 2^(31 + s) / page_size rounded up, s = ceil(log2 page_size): exact for keys below 2^31
  int s = 0;
  while ((1 << s) < d.page_size) ++s;
  p.page_shift = s;
  p.page_mul = (uint32_t)((((uint64_t)1 << (31 + s)) + d.page_size - 1) / d.page_size);
  p.c = d.softmax_scale * 1.4426950408889634f /* log2(e) */; p.causal = d.causal != 0;
  p.counters = static_cast<uint32_t*>(workspace);
  p.parts = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + kWsHeadBytes);
  p.slot_floats = pl.slot_floats;
  if (need > 0 && !(d.flags & LOONG_WORKSPACE_CLEAN))
    if (int rc = launch_clear_head(workspace, stream)) return rc;
  if (is_few(d)) launch_paged_few(p, d, (unsigned)pl.workgroups, stream);
  else launch_paged_many(p, d, dev.cus, (unsigned)pl.workgroups, stream);
  return check_launch("loong_paged_attn");
}

}  // extern "C"
