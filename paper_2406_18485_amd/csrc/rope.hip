// Norms of query and key heads with the position rotation, and their gradient: what lies between a projection and the
// first attention step, and between the last backward step and the projection's gradient.
//
// A group of lanes takes a token and walks over (a share of) its heads: the cosines and sines, some ten instructions a pair, five of
// them in 64 bits, are formed once for all of them.  Bound by HBM: forward 2 e bytes per element (e: its size), backward 2 e + 4.  Inputs that
// are in no cache: a prompt of 4096 tokens of 64 heads of 128, 134 MB, 23 us (5.7 TB/s; a plain elementwise pass reaches 5.3 at that
// size); the 1M-token shard's rows, 32768 tokens of 5 heads, forward 84 MB 17 us, backward 168 MB 35 us and 4 for the weights.
#include <hip/hip_runtime.h>

#include <cmath>

#include "loong_internal.h"
#include "rope_row.h"

namespace loong {
namespace {

constexpr int kRopeThreads = 256;

struct RopeParams {
  RopeRow row;
  const void *x[2];              // q, k
  const float* w[2];
  const int32_t* positions;
  void* y[2];                    // forward: rotated rows; backward: dq, dk
  const float* g[2];             // backward: gradients of the rotated rows
  int64_t xs[2][3], ys[2][3];    // strides of x (and of dq, dk); of the rotated rows (and their gradients)
  int64_t tokens;                // batch * len
  int32_t len, chunk_len, chunk[2];
  int32_t heads[2];
  int32_t heads_per_group;       // heads that a group of lanes walks over
  int64_t token_blocks;
  int32_t bwd_heads[2], bwd_blocks[2], bwd_wgs_q;   // backward: heads and workgroups of a share; the first so many workgroups are q's
  float* partial;                // backward: sums over a workgroup's rows, [workgroup][head_dim], or NULL
  int32_t head_dim;
};

__device__ __forceinline__ int64_t position_of(const RopeParams& p, int64_t token, int b, int t) {
  if (p.positions) return p.positions[token];
  if (p.chunk_len == 0) return t;
  const int half = t >= p.chunk_len;
  return (int64_t)(half ? p.chunk[1] : p.chunk[0]) * p.chunk_len + (t - half * p.chunk_len);
}

template <class E, bool INTER>
__global__ __launch_bounds__(kRopeThreads) void rope_fwd_kernel(const RopeParams p) {
  typedef typename StorageOf<E>::type T;
  constexpr int V = kRopeVec<E>, AT_ONCE = 4;
  const int s = threadIdx.x & ((1 << p.row.lg) - 1);
  const int64_t token = (int64_t)blockIdx.x * (kRopeThreads >> p.row.lg) + (threadIdx.x >> p.row.lg);
  if (token >= p.tokens) return;
  const int b = (int)(token / p.len), t = (int)(token - (int64_t)b * p.len);
  RopeLane<E, INTER> lane(p.row, s);
  const int64_t pos = position_of(p, token, b, t);
  const int h_lo = blockIdx.y * p.heads_per_group, h_hi = min(h_lo + p.heads_per_group, p.heads[0] + p.heads[1]);
  bool turned = false;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const int from = which ? p.heads[0] : 0;
    const int lo = max(h_lo, from) - from, hi = min(h_hi, from + p.heads[which]) - from;
    if (lo >= hi) continue;
    float w[2 * V];
    const T* x = (const T*)p.x[which] + b * p.xs[which][0] + t * p.xs[which][2];
    T* y = (T*)p.y[which] + b * p.ys[which][0] + t * p.ys[which][2];
    for (int h = lo; h < hi; h += AT_ONCE) {
      uint4 pa[AT_ONCE], pb[AT_ONCE];
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        const T* row = x + (int64_t)min(h + j, hi - 1) * p.xs[which][1];
        pa[j] = *reinterpret_cast<const uint4*>(row + lane.a);
        pb[j] = *reinterpret_cast<const uint4*>(row + lane.b);
      }
      if (h == lo && p.row.norm) lane.weights(p.w[which], w);
      if (!turned) lane.turn(p.row, s, pos);   // (while the first rows are on their way)
      turned = true;
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        if (h + j >= hi) break;
        lane.forward(p.row, w, pa[j], pb[j]);
        T* row = y + (int64_t)(h + j) * p.ys[which][1];
        if (lane.holds) {
          store_streaming(row + lane.a, pa[j]);
          store_streaming(row + lane.b, pb[j]);
        }
      }
    }
  }
}

// dx = r (w g - x r mean(w g x r)), g the gradient rotated back; a weight's gradient is the sum of g x r over all rows.  (Every factor is
// of a normal size that way: r^3 alone passes the largest float at rows of rms 1e-13, with an eps of 0.)
// A workgroup takes heads of q or of k and walks over token blocks, the next row's loads in flight while one is computed (48 us instead
// of the 35 above without, and with heads of both in a workgroup); its sums go to the workspace, and the kernel behind this one adds them up in order.
template <class E, bool INTER>
__global__ __launch_bounds__(kRopeThreads) void rope_bwd_kernel(const RopeParams p) {
  typedef typename StorageOf<E>::type T;
  constexpr int V = kRopeVec<E>;
  __shared__ float sums[kRopeThreads / 64][64][2 * V];
  const int lanes = 1 << p.row.lg, s = threadIdx.x & (lanes - 1);
  RopeLane<E, INTER> lane(p.row, s);
  const int which = (int)blockIdx.x >= p.bwd_wgs_q, wg = blockIdx.x - (which ? p.bwd_wgs_q : 0), blocks = p.bwd_blocks[which];
  const int share = wg / blocks, lo = share * p.bwd_heads[which], hi = min(lo + p.bwd_heads[which], p.heads[which]);
  const int64_t* const xs = p.xs[which];
  const int64_t* const ys = p.ys[which];
  float w[2 * V], dw[2 * V];
  if (p.row.norm) lane.weights(p.w[which], w);
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) dw[i] = 0.f;
  // one row of a token: where it is, and what is loaded of it
  struct Row {
    int64_t x, g;
    uint4 xa, xb;
    float4 v[V / 2];
  };
  const int per = kRopeThreads >> p.row.lg, group = threadIdx.x >> p.row.lg;
  int64_t block = wg - share * blocks, token = block * per + group;
  int h = lo;
  auto load = [&](int64_t token, int h) {
    const int b = (int)(token / p.len), t = (int)(token - (int64_t)b * p.len);
    Row r;
    r.x = b * xs[0] + h * xs[1] + t * xs[2];
    r.g = b * ys[0] + h * ys[1] + t * ys[2];
    const float* grow = p.g[which] + r.g;
#pragma unroll
    for (int i = 0; i < 2 * V; i += 4) r.v[i / 4] = *reinterpret_cast<const float4*>(grow + (i < V ? lane.a + i : lane.b + i - V));
    if (p.row.norm) {
      const T* row = (const T*)p.x[which] + r.x;
      r.xa = *reinterpret_cast<const uint4*>(row + lane.a);
      r.xb = *reinterpret_cast<const uint4*>(row + lane.b);
    }
    return r;
  };
  Row next;
  if (token < p.tokens) next = load(token, h);
  while (token < p.tokens) {   // (past it in a last block of few tokens, and then in every later one)
    const Row cur = next;
    if (h == lo) {
      const int b = (int)(token / p.len);
      lane.turn(p.row, s, position_of(p, token, b, (int)(token - (int64_t)b * p.len)));
    }
    if (++h == hi) {
      h = lo;
      block += blocks;
      token = block * per + group;
    }
    if (token < p.tokens) next = load(token, h);
    float gy[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; i += 4) {
      gy[i] = cur.v[i / 4].x; gy[i + 1] = cur.v[i / 4].y; gy[i + 2] = cur.v[i / 4].z; gy[i + 3] = cur.v[i / 4].w;
    }
    lane.rotate_back(gy);
    if (p.row.norm) {
      float xv[2 * V];
      unpack16<E>(cur.xa, xv);
      unpack16<E>(cur.xb, xv + V);
      // both sums of the row at once
      float sq = 0.f, dot = 0.f;
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        sq += xv[i] * xv[i];
        dot += gy[i] * w[i] * xv[i];
      }
      lane.row_sums(p.row, sq, dot);
      const float inv = rsqrtf(sq * p.row.inv_d + p.row.eps), mean = dot * inv * p.row.inv_d;
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) {
        const float hat = xv[i] * inv;
        dw[i] += gy[i] * hat;
        gy[i] = (gy[i] * w[i] - hat * mean) * inv;
      }
    }
    T* row = (T*)p.y[which] + cur.x;
    if (lane.holds) {
      store_streaming(row + lane.a, pack16<E>(gy));
      store_streaming(row + lane.b, pack16<E>(gy + V));
    }
  }
  if (!p.partial) return;
  // sums over the workgroup's groups: across a wave by exchange, across the waves through LDS, in a fixed order
  const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
  float* mine = p.partial + (int64_t)blockIdx.x * p.head_dim;
#pragma unroll
  for (int i = 0; i < 2 * V; ++i) {
    float x = dw[i];
    for (int m = 32; m >= lanes; m >>= 1) x += __shfl_xor(x, m, 64);
    if (l < lanes) sums[wave][l][i] = x;
  }
  __syncthreads();
  if (threadIdx.x < lanes && lane.holds) {
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) {
      float x = 0.f;
#pragma unroll
      for (int k = 0; k < kRopeThreads / 64; ++k) x += sums[k][s][i];
      mine[i < V ? lane.a + i : lane.b + i - V] = x;
    }
  }
}

// The workgroups' sums (those of q first), added up: 16 columns a workgroup, 64 threads a column.  Bound by the chain of loads:
// one in 64 of them each, eight at a time.  (16 threads a column: 14 us for 1024 sums.)
constexpr int kWeightThreads = 1024;
__global__ __launch_bounds__(kWeightThreads) void rope_weight_kernel(const float* partial, int nq, int nk, int head_dim, float* dwq, float* dwk) {
  __shared__ float sums[64][17];
  const int c = threadIdx.x & 15, part = threadIdx.x >> 4, at = blockIdx.x * 16 + c;
  const int which = at >= head_dim, col = at - which * head_dim, n = which ? nk : nq;
  const float* from = partial + (int64_t)(which ? nq : 0) * head_dim + col;
  float x = 0.f;
  for (int i = part; i < n; i += 64 * 8) {
    float y[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) y[k] = i + 64 * k < n ? from[(int64_t)(i + 64 * k) * head_dim] : 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) x += y[k];
  }
  sums[part][c] = x;
  __syncthreads();
  if (part) return;
  x = 0.f;
#pragma unroll
  for (int k = 0; k < 64; ++k) x += sums[k][c];
  float* dw = which ? dwk : dwq;
  if (dw) dw[col] = x;
}

int check_rope(const loong_rope_desc* d) {
  if (!d) return fail(LOONG_E_NULL, "descriptor is NULL");
  if (d->dtype != LOONG_BF16 && d->dtype != LOONG_FP32 && d->dtype != LOONG_FP16)
    return fail(LOONG_E_DTYPE, "dtype %d is none of LOONG_BF16, LOONG_FP32, LOONG_FP16", d->dtype);
  if (d->batch < 0 || d->len < 0 || d->n_q_heads < 0 || d->n_kv_heads < 0 || (int64_t)d->n_q_heads + d->n_kv_heads < 1)
    return fail(LOONG_E_SHAPE, "negative size or no heads (batch %d, len %d, heads %d/%d)", d->batch, d->len, d->n_q_heads, d->n_kv_heads);
  if (d->n_q_heads > kMaxHeads || d->n_kv_heads > kMaxHeads)
    return fail(LOONG_E_UNSUPPORTED, "heads %d/%d: %d of either at most", d->n_q_heads, d->n_kv_heads, kMaxHeads);
  if (d->head_dim < 16 || d->head_dim > 256 || d->head_dim % 16 != 0)
    return fail(LOONG_E_UNSUPPORTED, "head_dim %d is not a multiple of 16 up to 256", d->head_dim);
  if (d->rot_dim < 0 || d->rot_dim > d->head_dim || d->rot_dim % 16 != 0)
    return fail(LOONG_E_UNSUPPORTED, "rot_dim %d is not a multiple of 16 in [0, head_dim %d]", d->rot_dim, d->head_dim);
  if (d->flags & ~(LOONG_QK_NORM | LOONG_ROPE_INTERLEAVED)) return fail(LOONG_E_UNSUPPORTED, "flags %d: LOONG_QK_NORM, LOONG_ROPE_INTERLEAVED only", d->flags);
  if ((d->flags & LOONG_QK_NORM) && !(std::isfinite(d->eps) && d->eps >= 0.f)) return fail(LOONG_E_SHAPE, "eps must be finite and not negative");
  if (d->chunk_len != 0 && (d->chunk_len < 0 || (int64_t)d->chunk_len * 2 != d->len))
    return fail(LOONG_E_SHAPE, "zigzag positions need len == 2*chunk_len (got %d, %d)", d->len, d->chunk_len);
  if (d->chunk_len != 0 && (d->chunk[0] < 0 || d->chunk[1] < 0)) return fail(LOONG_E_SHAPE, "chunk ids must be non-negative");
  const int64_t* strides[4] = {d->q_stride, d->k_stride, d->q_out_stride, d->k_out_stride};
  const char* names[4] = {"q_stride", "k_stride", "q_out_stride", "k_out_stride"};
  const int vec = d->dtype == LOONG_FP32 ? 4 : 8;
  for (int t = 0; t < 4; ++t) {
    if ((t & 1 ? d->n_kv_heads : d->n_q_heads) == 0) continue;
    for (int i = 0; i < 3; ++i) {
      if (strides[t][i] < 0 || strides[t][i] > ((int64_t)1 << 48)) return fail(LOONG_E_SHAPE, "%s[%d] is negative or too large", names[t], i);
      if (strides[t][i] % vec != 0)
        return fail(LOONG_E_ALIGN, "%s[%d] = %lld is not a multiple of %d elements", names[t], i, (long long)strides[t][i], vec);
    }
  }
  if ((int64_t)d->batch * d->len > ((int64_t)1 << 31) - 1) return fail(LOONG_E_UNSUPPORTED, "more than 2^31 - 1 tokens");
  return LOONG_OK;
}

// the rows of a result of q's or k's heads, by its strides
int check_rope_result(const loong_rope_desc& d, const char* name, const int64_t* stride, int heads) {
  const int64_t n[3] = {d.batch, heads, d.len};
  if (d.batch == 0 || d.len == 0 || heads == 0) return LOONG_OK;
  for (int i = 0; i < 3; ++i)
    if (!apart(stride[i], n[i], d.head_dim)) return fail(LOONG_E_SHAPE, "%s[%d] = %lld: rows of a result lie on each other", name, i, (long long)stride[i]);
  return LOONG_OK;
}

// Forward: token blocks x shares of the heads; a group of lanes takes so many heads that the launch still has some `kFwdPerCu`
// workgroups for every unit.  Backward: a workgroup has heads of q or of k and walks over every so-manieth token block; there are as
// many of either as gives all of them equal work and every unit about `kBwdPerCu`, what its registers have room for.
constexpr int kFwdPerCu = 4, kBwdPerCu = 3;
struct RopePlan {
  int64_t token_blocks;
  int heads_per_group, shares;
  struct { int heads_per_group, shares; int64_t blocks; } bwd[2];   // q, k: `blocks` workgroups a share
  int64_t bwd_workgroups(int which) const { return bwd[which].shares * bwd[which].blocks; }
};
RopePlan plan_rope(const loong_rope_desc& d, const RopeRow& r, int cus) {
  RopePlan p{};
  const int64_t tokens = (int64_t)d.batch * d.len, per = kRopeThreads >> r.lg;
  const int heads[3] = {d.n_q_heads, d.n_kv_heads, d.n_q_heads + d.n_kv_heads};
  p.token_blocks = (tokens + per - 1) / per;
  const int64_t rows = p.token_blocks * heads[2];   // of lane groups: rows that a workgroup handles at a time
  const int64_t hpg = (rows + kFwdPerCu * (int64_t)cus - 1) / (kFwdPerCu * (int64_t)cus);
  p.heads_per_group = hpg < 1 ? 1 : hpg > heads[2] ? heads[2] : (int)hpg;
  p.shares = (heads[2] + p.heads_per_group - 1) / p.heads_per_group;
  const int64_t each = (rows + kBwdPerCu * (int64_t)cus - 1) / (kBwdPerCu * (int64_t)cus);   // rows a workgroup
  for (int k = 0; k < 2; ++k) {
    if (heads[k] == 0 || rows == 0) continue;
    p.bwd[k].heads_per_group = each > heads[k] ? heads[k] : (int)each;
    p.bwd[k].shares = (heads[k] + p.bwd[k].heads_per_group - 1) / p.bwd[k].heads_per_group;
    const int64_t blocks_each = (each + p.bwd[k].heads_per_group - 1) / p.bwd[k].heads_per_group;
    p.bwd[k].blocks = (p.token_blocks + blocks_each - 1) / blocks_each;
  }
  return p;
}

RopeRow row_of(const loong_rope_desc& d, const float* inv_freq) {
  return make_rope_row(d.head_dim, d.rot_dim, d.dtype == LOONG_FP32 ? 4 : 8, (d.flags & LOONG_QK_NORM) != 0, d.eps, inv_freq);
}

int64_t rope_workspace(const loong_rope_desc& d, int cus) {
  if (!(d.flags & LOONG_QK_NORM)) return 0;
  const RopePlan pl = plan_rope(d, row_of(d, nullptr), cus);
  return (pl.bwd_workgroups(0) + pl.bwd_workgroups(1)) * d.head_dim * 4;
}

// what both calls ask of their tensors; `names` of q and of its other tensors
int check_rope_tensors(const loong_rope_desc& d, const char* what, const float* inv_freq, const int32_t* positions, const float* const w[2],
                       const void* const q[4], const void* const k[4], int n) {
  if (d.rot_dim > 0 && !inv_freq) return fail(LOONG_E_NULL, "%s: NULL inv_freq", what);
  for (int i = 0; i < n; ++i) {
    if ((d.n_q_heads > 0 && !q[i]) || (d.n_kv_heads > 0 && !k[i])) return fail(LOONG_E_NULL, "%s: NULL tensor", what);
    if ((d.n_q_heads > 0 && !aligned16(q[i])) || (d.n_kv_heads > 0 && !aligned16(k[i]))) return fail(LOONG_E_ALIGN, "%s: tensor not 16-byte aligned", what);
  }
  if (!aligned16(w[0]) || !aligned16(w[1]) || !aligned16(inv_freq)) return fail(LOONG_E_ALIGN, "%s: weights or inv_freq not 16-byte aligned", what);
  if ((reinterpret_cast<uintptr_t>(positions)) & 3) return fail(LOONG_E_ALIGN, "%s: positions not 4-byte aligned", what);
  return LOONG_OK;
}

RopeParams params_of(const loong_rope_desc& d, const RopePlan& pl, const float* inv_freq, const int32_t* positions) {
  RopeParams p{};
  p.row = row_of(d, inv_freq);
  p.positions = positions;
  for (int i = 0; i < 3; ++i) {
    p.xs[0][i] = d.q_stride[i]; p.xs[1][i] = d.k_stride[i];
    p.ys[0][i] = d.q_out_stride[i]; p.ys[1][i] = d.k_out_stride[i];
  }
  p.tokens = (int64_t)d.batch * d.len;
  p.len = d.len; p.chunk_len = d.chunk_len; p.chunk[0] = d.chunk[0]; p.chunk[1] = d.chunk[1];
  p.heads[0] = d.n_q_heads; p.heads[1] = d.n_kv_heads;
  p.token_blocks = pl.token_blocks; p.head_dim = d.head_dim;
  return p;
}

template <class E>
void launch_rope_fwd(const RopeParams& p, dim3 grid, bool inter, hipStream_t st) {
  if (inter) rope_fwd_kernel<E, true><<<grid, dim3(kRopeThreads), 0, st>>>(p);
  else rope_fwd_kernel<E, false><<<grid, dim3(kRopeThreads), 0, st>>>(p);
}
template <class E>
void launch_rope_bwd(const RopeParams& p, dim3 grid, bool inter, hipStream_t st) {
  if (inter) rope_bwd_kernel<E, true><<<grid, dim3(kRopeThreads), 0, st>>>(p);
  else rope_bwd_kernel<E, false><<<grid, dim3(kRopeThreads), 0, st>>>(p);
}

}  // namespace
}  // namespace loong

using namespace loong;

extern "C" {

int loong_qk_rope_fwd(const loong_rope_desc* desc, const void* q, const void* k, const float* q_weight, const float* k_weight,
                      const float* inv_freq, const int32_t* positions, void* q_out, void* k_out, void* stream) {
  clear_error();
  if (int rc = check_rope(desc)) return rc;
  const float* w[2] = {q_weight, k_weight};
  const void *qs[4] = {q, q_out}, *ks[4] = {k, k_out};
  if (int rc = check_rope_tensors(*desc, "loong_qk_rope_fwd", inv_freq, positions, w, qs, ks, 2)) return rc;
  if (int rc = check_rope_result(*desc, "q_out_stride", desc->q_out_stride, desc->n_q_heads)) return rc;
  if (int rc = check_rope_result(*desc, "k_out_stride", desc->k_out_stride, desc->n_kv_heads)) return rc;
  const RopePlan pl = plan_rope(*desc, row_of(*desc, nullptr), planning_cus());
  if (pl.token_blocks == 0) return LOONG_OK;
  if (pl.shares > 65535 || !launch_fits(pl.token_blocks * pl.shares, kRopeThreads)) return fail(LOONG_E_UNSUPPORTED, "loong_qk_rope_fwd: grid too large");
  RopeParams p = params_of(*desc, pl, inv_freq, positions);
  p.heads_per_group = pl.heads_per_group;
  p.x[0] = q; p.x[1] = k; p.w[0] = q_weight; p.w[1] = k_weight; p.y[0] = q_out; p.y[1] = k_out;
  const dim3 grid((unsigned)pl.token_blocks, (unsigned)pl.shares);
  const bool inter = (desc->flags & LOONG_ROPE_INTERLEAVED) != 0;
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (desc->dtype == LOONG_BF16) launch_rope_fwd<Bf16>(p, grid, inter, st);
  else if (desc->dtype == LOONG_FP16) launch_rope_fwd<Fp16>(p, grid, inter, st);
  else launch_rope_fwd<float>(p, grid, inter, st);
  return check_launch("loong_qk_rope_fwd");
}

int loong_qk_rope_workspace_bytes(const loong_rope_desc* desc, int64_t* bytes) {
  clear_error();
  if (!bytes) return fail(LOONG_E_NULL, "loong_qk_rope_workspace_bytes: NULL result");
  if (int rc = check_rope(desc)) return rc;
  *bytes = rope_workspace(*desc, planning_cus());
  return LOONG_OK;
}

int loong_qk_rope_bwd(const loong_rope_desc* desc, const void* q, const void* k, const float* q_weight, const float* k_weight,
                      const float* inv_freq, const int32_t* positions, const float* d_q_out, const float* d_k_out, void* dq, void* dk,
                      float* dq_weight, float* dk_weight, void* workspace, int64_t workspace_bytes, void* stream) {
  clear_error();
  if (int rc = check_rope(desc)) return rc;
  const float* w[2] = {q_weight, k_weight};
  const void *qs[4] = {q, d_q_out, dq}, *ks[4] = {k, d_k_out, dk};
  if (int rc = check_rope_tensors(*desc, "loong_qk_rope_bwd", inv_freq, positions, w, qs, ks, 3)) return rc;
  if (int rc = check_rope_result(*desc, "q_stride (of dq)", desc->q_stride, desc->n_q_heads)) return rc;
  if (int rc = check_rope_result(*desc, "k_stride (of dk)", desc->k_stride, desc->n_kv_heads)) return rc;
  const bool norm = (desc->flags & LOONG_QK_NORM) != 0, sums = dq_weight || dk_weight;
  if (sums && !norm) return fail(LOONG_E_UNSUPPORTED, "loong_qk_rope_bwd: gradients of weights without LOONG_QK_NORM");
  if ((dq_weight && desc->n_q_heads == 0) || (dk_weight && desc->n_kv_heads == 0))
    return fail(LOONG_E_UNSUPPORTED, "loong_qk_rope_bwd: gradient of the weights of heads that are not there");
  if ((reinterpret_cast<uintptr_t>(dq_weight) | reinterpret_cast<uintptr_t>(dk_weight)) & 3) return fail(LOONG_E_ALIGN, "loong_qk_rope_bwd: weight gradient not 4-byte aligned");
  const int cus = planning_cus();
  const RopePlan pl = plan_rope(*desc, row_of(*desc, nullptr), cus);
  const int64_t need = rope_workspace(*desc, cus);
  if (sums && need > 0) {
    if (!workspace) return fail(LOONG_E_NULL, "loong_qk_rope_bwd: NULL workspace");
    if (!aligned16(workspace)) return fail(LOONG_E_ALIGN, "loong_qk_rope_bwd: workspace not 16-byte aligned");
    if (workspace_bytes < need)
      return fail(LOONG_E_SHAPE, "loong_qk_rope_bwd: workspace of %lld bytes, %lld are needed", (long long)workspace_bytes, (long long)need);
  }
  const int64_t nq = pl.bwd_workgroups(0), nk = pl.bwd_workgroups(1);
  if (!launch_fits(nq + nk, kRopeThreads)) return fail(LOONG_E_UNSUPPORTED, "loong_qk_rope_bwd: grid too large");
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (pl.token_blocks > 0) {
    RopeParams p = params_of(*desc, pl, inv_freq, positions);
    for (int i = 0; i < 2; ++i) { p.bwd_heads[i] = pl.bwd[i].heads_per_group; p.bwd_blocks[i] = (int)pl.bwd[i].blocks; }
    p.bwd_wgs_q = (int)nq;
    p.x[0] = q; p.x[1] = k; p.w[0] = q_weight; p.w[1] = k_weight; p.y[0] = dq; p.y[1] = dk; p.g[0] = d_q_out; p.g[1] = d_k_out;
    p.partial = sums ? static_cast<float*>(workspace) : nullptr;
    const dim3 grid((unsigned)(nq + nk));
    const bool inter = (desc->flags & LOONG_ROPE_INTERLEAVED) != 0;
    if (desc->dtype == LOONG_BF16) launch_rope_bwd<Bf16>(p, grid, inter, st);
    else if (desc->dtype == LOONG_FP16) launch_rope_bwd<Fp16>(p, grid, inter, st);
    else launch_rope_bwd<float>(p, grid, inter, st);
    if (int rc = check_launch("loong_qk_rope_bwd")) return rc;
  }
  if (!sums) return LOONG_OK;
  rope_weight_kernel<<<dim3((unsigned)(2 * desc->head_dim / 16)), dim3(kWeightThreads), 0, st>>>(
      static_cast<const float*>(workspace), (int)nq, (int)nk, desc->head_dim, dq_weight, dk_weight);
  return check_launch("loong_qk_rope_bwd (weights)");
}

}  // extern "C"
