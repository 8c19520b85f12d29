// Norms of query and key heads with the position rotation, and their gradient: what lies between a projection and the
// first attention step, and between the last backward step and the projection's gradient.
//
// A group of lanes takes a token and walks over (a share of) its heads: the cosines and sines, some 40 instructions a pair,
// are formed once for all of them.  Bound by HBM: forward 2 e bytes per element (e: its size), backward 2 e + 4.
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
  float* partial;                // backward: sums over a workgroup's rows, [workgroup][q, k][head_dim], or NULL
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
  lane.turn(p.row, s, position_of(p, token, b, t));
  const int h_lo = blockIdx.y * p.heads_per_group, h_hi = min(h_lo + p.heads_per_group, p.heads[0] + p.heads[1]);
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const int from = which ? p.heads[0] : 0;
    const int lo = max(h_lo, from) - from, hi = min(h_hi, from + p.heads[which]) - from;
    if (lo >= hi) continue;
    float w[2 * V];
    if (p.row.norm) lane.weights(p.w[which], w);
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
#pragma unroll
      for (int j = 0; j < AT_ONCE; ++j) {
        if (h + j >= hi) break;
        lane.forward(p.row, w, pa[j], pb[j]);
        T* row = y + (int64_t)(h + j) * p.ys[which][1];
        if (lane.holds) {
          *reinterpret_cast<uint4*>(row + lane.a) = pa[j];
          *reinterpret_cast<uint4*>(row + lane.b) = pb[j];
        }
      }
    }
  }
}

// dx = r (w g) - x r^3 mean(w g x), g the gradient rotated back; a weight's gradient is the sum of g x r over all rows.
// A workgroup walks over token blocks; its sums go to the workspace, and the kernel behind this one adds them up in order.
template <class E, bool INTER>
__global__ __launch_bounds__(kRopeThreads) void rope_bwd_kernel(const RopeParams p) {
  typedef typename StorageOf<E>::type T;
  constexpr int V = kRopeVec<E>;
  __shared__ float sums[kRopeThreads / 64][64][2 * V];
  const int lanes = 1 << p.row.lg, s = threadIdx.x & (lanes - 1);
  RopeLane<E, INTER> lane(p.row, s);
  const int h_lo = blockIdx.y * p.heads_per_group, h_hi = min(h_lo + p.heads_per_group, p.heads[0] + p.heads[1]);
  float dw[2][2 * V];
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) dw[which][i] = 0.f;
  for (int64_t block = blockIdx.x; block < p.token_blocks; block += gridDim.x) {
    const int64_t token = block * (kRopeThreads >> p.row.lg) + (threadIdx.x >> p.row.lg);
    if (token >= p.tokens) break;   // (only in the last block)
    const int b = (int)(token / p.len), t = (int)(token - (int64_t)b * p.len);
    lane.turn(p.row, s, position_of(p, token, b, t));
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const int from = which ? p.heads[0] : 0;
      const int lo = max(h_lo, from) - from, hi = min(h_hi, from + p.heads[which]) - from;
      if (lo >= hi) continue;
      float w[2 * V];
      if (p.row.norm) lane.weights(p.w[which], w);
      const T* x = (const T*)p.x[which] + b * p.xs[which][0] + t * p.xs[which][2];
      const float* g = p.g[which] + b * p.ys[which][0] + t * p.ys[which][2];
      T* dx = (T*)p.y[which] + b * p.xs[which][0] + t * p.xs[which][2];
      for (int h = lo; h < hi; ++h) {
        float gy[2 * V];
        const float* grow = g + (int64_t)h * p.ys[which][1];
#pragma unroll
        for (int i = 0; i < 2 * V; i += 4) {
          const float4 v4 = *reinterpret_cast<const float4*>(grow + (i < V ? lane.a + i : lane.b + i - V));
          gy[i] = v4.x; gy[i + 1] = v4.y; gy[i + 2] = v4.z; gy[i + 3] = v4.w;
        }
        lane.rotate_back(gy);
        if (p.row.norm) {
          float xv[2 * V];
          const T* row = x + (int64_t)h * p.xs[which][1];
          unpack16<E>(*reinterpret_cast<const uint4*>(row + lane.a), xv);
          unpack16<E>(*reinterpret_cast<const uint4*>(row + lane.b), xv + V);
          const float inv = lane.rms(p.row, xv);
          float dot = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            dw[which][i] += gy[i] * (xv[i] * inv);
            gy[i] *= w[i];
            dot += gy[i] * xv[i];
          }
          const float c = lane.row_sum(p.row, dot) * p.row.inv_d * (inv * inv * inv);
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) gy[i] = gy[i] * inv - xv[i] * c;
        }
        T* row = dx + (int64_t)h * p.xs[which][1];
        if (lane.holds) {
          *reinterpret_cast<uint4*>(row + lane.a) = pack16<E>(gy);
          *reinterpret_cast<uint4*>(row + lane.b) = pack16<E>(gy + V);
        }
      }
    }
  }
  if (!p.partial) return;
  // sums over the workgroup's groups: across a wave by exchange, across the waves through LDS, in a fixed order
  const int wave = threadIdx.x >> 6, l = threadIdx.x & 63;
  float* mine = p.partial + ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 * p.head_dim;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) {
      float x = dw[which][i];
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
        mine[which * p.head_dim + (i < V ? lane.a + i : lane.b + i - V)] = x;
      }
    }
    __syncthreads();
  }
}

// The workgroups' sums, added up: 16 columns a workgroup, 16 threads a column, each over every 16th of them.
__global__ __launch_bounds__(256) void rope_weight_kernel(const float* partial, int n, int head_dim, float* dwq, float* dwk) {
  __shared__ float sums[16][17];
  const int c = threadIdx.x & 15, part = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
  float x = 0.f;
  for (int i = part; i < n; i += 16) x += partial[(int64_t)i * 2 * head_dim + col];
  sums[part][c] = x;
  __syncthreads();
  if (part) return;
  x = 0.f;
#pragma unroll
  for (int k = 0; k < 16; ++k) x += sums[k][c];
  float* dw = col < head_dim ? dwq : dwk;
  if (dw) dw[col < head_dim ? col : col - head_dim] = x;
}

int check_rope(const loong_rope_desc* d) {
  if (!d) return fail(LOONG_E_NULL, "descriptor is NULL");
  if (d->dtype != LOONG_BF16 && d->dtype != LOONG_FP32 && d->dtype != LOONG_FP16)
    return fail(LOONG_E_DTYPE, "dtype %d is none of LOONG_BF16, LOONG_FP32, LOONG_FP16", d->dtype);
  if (d->batch < 0 || d->len < 0 || d->n_q_heads < 0 || d->n_kv_heads < 0 || (int64_t)d->n_q_heads + d->n_kv_heads < 1)
    return fail(LOONG_E_SHAPE, "negative size or no heads (batch %d, len %d, heads %d/%d)", d->batch, d->len, d->n_q_heads, d->n_kv_heads);
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

// Token blocks x shares of the heads.  A group of lanes takes so many heads that the launch still has some 16 waves for
// every unit; the backward's token blocks are walked over by at most four workgroups a unit, so that few sums are left.
struct RopePlan {
  int64_t token_blocks;
  int heads_per_group, shares;
  int64_t bwd_blocks;     // workgroups of a share
};
RopePlan plan_rope(const loong_rope_desc& d, const RopeRow& r, int cus) {
  RopePlan p{};
  const int64_t tokens = (int64_t)d.batch * d.len, per = kRopeThreads >> r.lg;
  const int heads = d.n_q_heads + d.n_kv_heads;
  p.token_blocks = (tokens + per - 1) / per;
  const int64_t hpg = p.token_blocks * heads / (4 * (int64_t)cus);
  p.heads_per_group = hpg < 1 ? 1 : hpg > heads ? heads : (int)hpg;
  p.shares = (heads + p.heads_per_group - 1) / p.heads_per_group;
  const int64_t most = (4 * (int64_t)cus + p.shares - 1) / p.shares;
  p.bwd_blocks = p.token_blocks < most ? p.token_blocks : most;
  return p;
}

RopeRow row_of(const loong_rope_desc& d, const float* inv_freq) {
  return make_rope_row(d.head_dim, d.rot_dim, d.dtype == LOONG_FP32 ? 4 : 8, (d.flags & LOONG_QK_NORM) != 0, d.eps, inv_freq);
}

int64_t rope_workspace(const loong_rope_desc& d, int cus) {
  if (!(d.flags & LOONG_QK_NORM)) return 0;
  const RopePlan pl = plan_rope(d, row_of(d, nullptr), cus);
  return pl.bwd_blocks * pl.shares * 2 * d.head_dim * 4;
}

// what both calls ask of their tensors; `names` of q and of its other tensors
int check_rope_tensors(const loong_rope_desc& d, const char* what, const float* inv_freq, const int32_t* positions, const float* const w[2],
                       const void* const q[4], const void* const k[4], int n) {
  if (d.rot_dim > 0 && !inv_freq) return fail(LOONG_E_NULL, "%s: NULL inv_freq", what);
  for (int i = 0; i < n; ++i) {
    if ((d.n_q_heads > 0 && !q[i]) || (d.n_kv_heads > 0 && !k[i])) return fail(LOONG_E_NULL, "%s: NULL tensor", what);
    if ((d.n_q_heads > 0 && !aligned16(q[i])) || (d.n_kv_heads > 0 && !aligned16(k[i]))) return fail(LOONG_E_ALIGN, "%s: tensor not 16-byte aligned", what);
  }
  if (!aligned16(w[0]) || !aligned16(w[1])) return fail(LOONG_E_ALIGN, "%s: weights not 16-byte aligned", what);
  if ((reinterpret_cast<uintptr_t>(inv_freq) | reinterpret_cast<uintptr_t>(positions)) & 3) return fail(LOONG_E_ALIGN, "%s: inv_freq or positions not 4-byte aligned", what);
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
  p.heads_per_group = pl.heads_per_group; p.token_blocks = pl.token_blocks; p.head_dim = d.head_dim;
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
  const RopePlan pl = plan_rope(*desc, row_of(*desc, nullptr), planning_cus());
  if (pl.token_blocks == 0) return LOONG_OK;
  if (pl.shares > 65535 || !launch_fits(pl.token_blocks * pl.shares, kRopeThreads)) return fail(LOONG_E_UNSUPPORTED, "loong_qk_rope_fwd: grid too large");
  RopeParams p = params_of(*desc, pl, inv_freq, positions);
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
  if (pl.shares > 65535 || !launch_fits(pl.bwd_blocks * pl.shares, kRopeThreads)) return fail(LOONG_E_UNSUPPORTED, "loong_qk_rope_bwd: grid too large");
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (pl.token_blocks > 0) {
    RopeParams p = params_of(*desc, pl, inv_freq, positions);
    p.x[0] = q; p.x[1] = k; p.w[0] = q_weight; p.w[1] = k_weight; p.y[0] = dq; p.y[1] = dk; p.g[0] = d_q_out; p.g[1] = d_k_out;
    p.partial = sums ? static_cast<float*>(workspace) : nullptr;
    const dim3 grid((unsigned)pl.bwd_blocks, (unsigned)pl.shares);
    const bool inter = (desc->flags & LOONG_ROPE_INTERLEAVED) != 0;
    if (desc->dtype == LOONG_BF16) launch_rope_bwd<Bf16>(p, grid, inter, st);
    else if (desc->dtype == LOONG_FP16) launch_rope_bwd<Fp16>(p, grid, inter, st);
    else launch_rope_bwd<float>(p, grid, inter, st);
    if (int rc = check_launch("loong_qk_rope_bwd")) return rc;
  }
  if (!sums) return LOONG_OK;
  rope_weight_kernel<<<dim3((unsigned)(2 * desc->head_dim / 16)), dim3(256), 0, st>>>(
      static_cast<const float*>(workspace), (int)(pl.bwd_blocks * pl.shares), desc->head_dim, dq_weight, dk_weight);
  return check_launch("loong_qk_rope_bwd (weights)");
}

}  // extern "C"
