// New tokens into a paged cache: keys normed and rotated, values as they are, and the queries beside them.
//
// A group of lanes takes a token, finds its sequence and slot, and walks over (a share of) its q, k and v heads; the norm and
// the rotation are those of rope_row.h.  Long prompts are bound by HBM, 2 e bytes per element of q and of k and v (16384 tokens of 32 + 2 x 8
// heads of 128: 403 MB in 63 us, some of it in the last-level cache); single tokens by the chain of loads from a token to its slot
// (seq_start, kv_len, page_table): 64 of them, 48 heads each, 4.4 us, of which a launch alone is 2.3.  Rows loaded four at a time and
// ahead of the chain were no faster (64 single tokens 4.4 -> 4.7 us, 2000 tokens 12.4 -> 14.3): the registers cost waves.
#include <hip/hip_runtime.h>

#include <cmath>

#include "loong_internal.h"
#include "rope_row.h"

namespace loong {

int check_paged(const loong_paged_desc* d, int flags) {
  if (!d) return fail(LOONG_E_NULL, "descriptor is NULL");
  if (d->dtype != LOONG_BF16 && d->dtype != LOONG_FP32 && d->dtype != LOONG_FP16)
    return fail(LOONG_E_DTYPE, "dtype %d is none of LOONG_BF16, LOONG_FP32, LOONG_FP16", d->dtype);
  if (d->dtype == LOONG_FP32) return fail(LOONG_E_UNSUPPORTED, "a paged cache holds LOONG_BF16 or LOONG_FP16");
  if (d->n_seqs < 0 || d->n_tokens < 0 || d->max_new < 0 || d->n_q_heads < 1 || d->n_kv_heads < 1 || d->n_pages < 0 || d->page_size < 1 ||
      d->max_pages < 0)
    return fail(LOONG_E_SHAPE, "negative size, zero heads or empty pages (n_seqs %d, n_tokens %d, max_new %d, heads %d/%d, n_pages %d, page_size %d, max_pages %d)",
                d->n_seqs, d->n_tokens, d->max_new, d->n_q_heads, d->n_kv_heads, d->n_pages, d->page_size, d->max_pages);
  if (d->n_q_heads % d->n_kv_heads != 0)
    return fail(LOONG_E_UNSUPPORTED, "n_q_heads %d is not a multiple of n_kv_heads %d", d->n_q_heads, d->n_kv_heads);
  if (d->n_q_heads > kMaxHeads) return fail(LOONG_E_UNSUPPORTED, "%d query heads: %d at most", d->n_q_heads, kMaxHeads);
  if (d->head_dim != 64 && d->head_dim != 128) return fail(LOONG_E_UNSUPPORTED, "a paged cache takes head_dim 64 or 128, got %d", d->head_dim);
  if (d->flags & ~flags) return fail(LOONG_E_UNSUPPORTED, "flags %d: this call takes %d", d->flags, flags);
  if (d->page_size > (1 << 24)) return fail(LOONG_E_UNSUPPORTED, "page_size %d is above 2^24", d->page_size);
  if ((int64_t)d->max_pages * d->page_size > (1 << 30)) return fail(LOONG_E_UNSUPPORTED, "more than 2^30 keys in a row of the page table");
  if (d->n_seqs > (1 << 20)) return fail(LOONG_E_UNSUPPORTED, "more than 2^20 sequences");
  if ((int64_t)d->n_tokens * d->n_q_heads > (1 << 30)) return fail(LOONG_E_UNSUPPORTED, "more than 2^30 query rows");
  const struct { const char* name; const int64_t* s; int n; } strides[] = {
      {"q_stride", d->q_stride, 2}, {"kv_stride", d->kv_stride, 2}, {"o_stride", d->o_stride, 2}, {"cache_stride", d->cache_stride, 3}};
  for (const auto& t : strides)
    for (int i = 0; i < t.n; ++i) {
      if (t.s[i] < 0 || t.s[i] > ((int64_t)1 << 40)) return fail(LOONG_E_SHAPE, "%s[%d] is negative or too large", t.name, i);
      if (t.s[i] % 8 != 0) return fail(LOONG_E_ALIGN, "%s[%d] = %lld is not a multiple of 8 elements", t.name, i, (long long)t.s[i]);
    }
  if (d->cache_stride[2] >= ((int64_t)1 << 31)) return fail(LOONG_E_UNSUPPORTED, "slot strides must be below 2^31 elements");
  if (d->table_stride < 0 || d->table_stride > ((int64_t)1 << 40)) return fail(LOONG_E_SHAPE, "table_stride is negative or too large");
  return LOONG_OK;
}

namespace {

constexpr int kAppendThreads = 256;

struct AppendParams {
  RopeRow row;
  const uint16_t *q, *k, *v;
  const float *wq, *wk;
  const int32_t *positions, *seq_start, *kv_len, *table;
  uint16_t *q_out, *k_cache, *v_cache;
  int64_t qs[2], kvs[2], os[2], cs[3], ts;
  int32_t n_seqs, n_tokens, hq, hkv, n_pages, page_size, max_pages;   // hq: 0 without q
  int32_t heads_per_group;
};

template <class E, bool INTER>
__global__ __launch_bounds__(kAppendThreads) void paged_append_kernel(const AppendParams p) {
  constexpr int V = kRopeVec<E>;
  const int lane_id = threadIdx.x & 63, lg = p.row.lg, s = threadIdx.x & ((1 << lg) - 1);
  const int first = blockIdx.x * (kAppendThreads >> lg) + ((threadIdx.x & ~63) >> lg);   // of this wave's tokens, which are consecutive
  const int mine = lane_id >> lg, token = first + mine;
  // the sequence of every token: how many of them end at or before it (empty ones among them), 64 at a time
  int b = 0;
  for (int base = 0; base < p.n_seqs; base += 64) {
    const int end = base + lane_id < p.n_seqs ? p.seq_start[base + lane_id + 1] : 0x7fffffff;
    for (int g = 0; g < 64 >> lg; ++g) {
      const int n = __popcll(__builtin_amdgcn_ballot_w64(end <= first + g));
      b += g == mine ? n : 0;
    }
  }
  if (token >= p.n_tokens || b >= p.n_seqs) return;
  const int start = max(p.seq_start[b], 0), n_new = min(p.seq_start[b + 1], p.n_tokens) - start;
  if (token < start) return;
  const int64_t slot = (int64_t)max(p.kv_len[b], 0) - n_new + (token - start);
  int64_t at = -1;   // where the token lies in the cache (elements), or nowhere
  if (slot >= 0 && slot < (int64_t)p.max_pages * p.page_size) {
    const uint32_t idx = (uint32_t)slot / (uint32_t)p.page_size, in = (uint32_t)slot - idx * (uint32_t)p.page_size;
    const int page = p.table[b * p.ts + idx];
    if (page >= 0 && page < p.n_pages) at = page * p.cs[0] + in * p.cs[2];
  }
  RopeLane<E, INTER> lane(p.row, s);
  lane.turn(p.row, s, p.positions ? p.positions[token] : slot);
  const int h_lo = blockIdx.y * p.heads_per_group, h_hi = min(h_lo + p.heads_per_group, p.hq + 2 * p.hkv);
  float wq[2 * V], wk[2 * V];
  if (p.row.norm) {
    lane.weights(p.wq, wq);
    lane.weights(p.wk, wk);
  }
  for (int h = h_lo; h < h_hi; ++h) {
    const bool is_q = h < p.hq, is_k = !is_q && h < p.hq + p.hkv;
    const int hk = h - p.hq - (is_k ? 0 : p.hkv);
    if (!is_q && at < 0) continue;
    const uint16_t* src = is_q ? p.q + token * p.qs[0] + h * p.qs[1] : (is_k ? p.k : p.v) + token * p.kvs[0] + hk * p.kvs[1];
    uint16_t* dst = is_q ? p.q_out + token * p.os[0] + h * p.os[1] : (is_k ? p.k_cache : p.v_cache) + at + hk * p.cs[1];
    uint4 pa = *reinterpret_cast<const uint4*>(src + lane.a), pb = *reinterpret_cast<const uint4*>(src + lane.b);
    if (is_q) lane.forward(p.row, wq, pa, pb);
    else if (is_k) lane.forward(p.row, wk, pa, pb);
    if (lane.holds) {
      store_streaming(dst + lane.a, pa);
      store_streaming(dst + lane.b, pb);
    }
  }
}

template <class E>
void launch_append(const AppendParams& p, dim3 grid, bool inter, hipStream_t st) {
  if (inter) paged_append_kernel<E, true><<<grid, dim3(kAppendThreads), 0, st>>>(p);
  else paged_append_kernel<E, false><<<grid, dim3(kAppendThreads), 0, st>>>(p);
}

}  // namespace
}  // namespace loong

using namespace loong;

extern "C" {

int loong_paged_append(const loong_paged_desc* desc, const void* q, const void* k, const void* v, const float* q_weight,
                       const float* k_weight, const float* inv_freq, const int32_t* positions, const int32_t* seq_start,
                       const int32_t* kv_len, const int32_t* page_table, void* q_out, void* k_cache, void* v_cache, void* stream) {
  clear_error();
  if (int rc = check_paged(desc, LOONG_QK_NORM | LOONG_ROPE_INTERLEAVED)) return rc;
  const loong_paged_desc& d = *desc;
  if (d.rot_dim < 0 || d.rot_dim > d.head_dim || d.rot_dim % 16 != 0)
    return fail(LOONG_E_UNSUPPORTED, "rot_dim %d is not a multiple of 16 in [0, head_dim %d]", d.rot_dim, d.head_dim);
  const bool norm = (d.flags & LOONG_QK_NORM) != 0;
  if (norm && !(std::isfinite(d.eps) && d.eps >= 0.f)) return fail(LOONG_E_SHAPE, "eps must be finite and not negative");
  if (!k || !v || !seq_start || !kv_len || !page_table || !k_cache || !v_cache || (d.rot_dim > 0 && !inv_freq) || !q != !q_out)
    return fail(LOONG_E_NULL, "loong_paged_append: NULL argument");
  for (const void* x : {q, k, v, (const void*)q_weight, (const void*)k_weight, (const void*)inv_freq, (const void*)q_out, (const void*)k_cache, (const void*)v_cache})
    if (!aligned16(x)) return fail(LOONG_E_ALIGN, "loong_paged_append: tensor not 16-byte aligned");
  for (const void* x : {(const void*)positions, (const void*)seq_start, (const void*)kv_len, (const void*)page_table})
    if (reinterpret_cast<uintptr_t>(x) & 3) return fail(LOONG_E_ALIGN, "loong_paged_append: table or inv_freq not 4-byte aligned");
  if (d.n_tokens == 0 || d.n_seqs == 0) return LOONG_OK;
  const int64_t cached[3] = {d.n_pages, d.n_kv_heads, d.page_size}, rows[2] = {d.n_tokens, d.n_q_heads};
  for (int i = 0; i < 3; ++i)
    if (!apart(d.cache_stride[i], cached[i], d.head_dim)) return fail(LOONG_E_SHAPE, "cache_stride[%d] = %lld: slots lie on each other", i, (long long)d.cache_stride[i]);
  for (int i = 0; i < 2 && q; ++i)
    if (!apart(d.o_stride[i], rows[i], d.head_dim)) return fail(LOONG_E_SHAPE, "o_stride[%d] = %lld: rows of a result lie on each other", i, (long long)d.o_stride[i]);
  AppendParams p{};
  p.row = make_rope_row(d.head_dim, d.rot_dim, 8, norm, d.eps, inv_freq);
  p.q = (const uint16_t*)q; p.k = (const uint16_t*)k; p.v = (const uint16_t*)v;
  p.wq = q_weight; p.wk = k_weight; p.positions = positions; p.seq_start = seq_start; p.kv_len = kv_len; p.table = page_table;
  p.q_out = (uint16_t*)q_out; p.k_cache = (uint16_t*)k_cache; p.v_cache = (uint16_t*)v_cache;
  for (int i = 0; i < 2; ++i) { p.qs[i] = d.q_stride[i]; p.kvs[i] = d.kv_stride[i]; p.os[i] = d.o_stride[i]; }
  for (int i = 0; i < 3; ++i) p.cs[i] = d.cache_stride[i];
  p.ts = d.table_stride;
  p.n_seqs = d.n_seqs; p.n_tokens = d.n_tokens; p.hq = q ? d.n_q_heads : 0; p.hkv = d.n_kv_heads;
  p.n_pages = d.n_pages; p.page_size = d.page_size; p.max_pages = d.max_pages;
  const int per = kAppendThreads >> p.row.lg, heads = p.hq + 2 * p.hkv;
  const int64_t blocks = ((int64_t)d.n_tokens + per - 1) / per;
  const int64_t hpg = blocks * heads / (4 * (int64_t)planning_cus());   // (as in plan_rope: some 16 waves a unit)
  p.heads_per_group = hpg < 1 ? 1 : hpg > heads ? heads : (int)hpg;
  const int shares = (heads + p.heads_per_group - 1) / p.heads_per_group;
  if (shares > 65535 || !launch_fits(blocks * shares, kAppendThreads)) return fail(LOONG_E_UNSUPPORTED, "loong_paged_append: grid too large");
  const dim3 grid((unsigned)blocks, (unsigned)shares);
  const bool inter = (d.flags & LOONG_ROPE_INTERLEAVED) != 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (d.dtype == LOONG_BF16) launch_append<Bf16>(p, grid, inter, st);
  else launch_append<Fp16>(p, grid, inter, st);
  return check_launch("loong_paged_append");
}

}  // extern "C"
