// Norm and rotation of one row (a head of a token), by a group of 2^lg lanes, for the kernels that take q and k from a
// projection: into the layout of the attention steps, or into a paged cache.
//
// A lane holds two 16-byte pieces of the row, V elements each, chosen so that both halves of every pair it rotates are its
// own: pieces s and s + rot/2 of the rotated part (pairs half of it apart), or 2 s and 2 s + 1 (neighbouring pairs, and
// what is not rotated).  Either way the lane's V pairs are numbers s V .. s V + V - 1, so one set of V cosines and sines serves
// all heads of a token.
#pragma once
#include <hip/hip_runtime.h>

#include "device_utils.h"

namespace loong {

template <class E>
constexpr int kRopeVec = std::is_same<E, float>::value ? 4 : 8;  // elements in 16 bytes

// 16 bytes that are written once and not read again by this kernel: past the caches' lines in use.  (A prompt of 4096 tokens, 64 heads
// of 128, 30.4 -> 23.6 us; the 1M-token shard's rows, forward and backward, 61.6 -> 57.7; 8000 tokens of 10 heads of 64, which caches
// would hold, 25.4 -> 24.1; 16384 tokens of 32 + 2 x 8 heads of 128 appended 89 -> 63, 64 single tokens the same.)
typedef uint32_t rope_u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store_streaming(void* p, uint4 v) {
  const rope_u32x4 x = {v.x, v.y, v.z, v.w};
  __builtin_nontemporal_store(x, static_cast<rope_u32x4*>(p));
}

struct RopeRow {
  int lg;          // log2 of the lanes per row
  int pieces2;     // lanes that hold elements: head_dim / (2 V)
  int rot2;        // those whose elements are rotated
  int norm;
  float eps, inv_d;
  const float* inv_freq;
};

template <class E>
__device__ __forceinline__ void unpack16(uint4 w, float* x) {
  if constexpr (std::is_same<E, float>::value) {
    x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
  } else {
    x[0] = E::lo(w.x); x[1] = E::hi(w.x); x[2] = E::lo(w.y); x[3] = E::hi(w.y);
    x[4] = E::lo(w.z); x[5] = E::hi(w.z); x[6] = E::lo(w.w); x[7] = E::hi(w.w);
  }
}
template <class E>
__device__ __forceinline__ uint4 pack16(const float* x) {
  if constexpr (std::is_same<E, float>::value)
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
  else
    return make_uint4(E::pack2(x[0], x[1]), E::pack2(x[2], x[3]), E::pack2(x[4], x[5]), E::pack2(x[6], x[7]));
}

// A lane's part of the rows: which pieces, and the factors of its pairs.
template <class E, bool INTER>
struct RopeLane {
  static constexpr int V = kRopeVec<E>;
  int a, b;              // element offsets of the two pieces
  bool holds;            // (of 2^lg lanes those past the row's end hold nothing)
  bool turns;            // its pairs are rotated.  (By 0 is not the same: infinity x 0 would make a NaN of its neighbour.)
  float cs[V], sn[V];

  __device__ __forceinline__ RopeLane(const RopeRow& r, int s) {
    holds = s < r.pieces2;
    turns = s < r.rot2;
    s = holds ? s : 0;
    const bool apart = !INTER && turns;
    a = (apart ? s : 2 * s) * V;
    b = (apart ? s + r.rot2 : 2 * s + 1) * V;
  }

  // The angle p f is reduced in 64 bits, in turns: at a position of a million its whole turns leave 32 bits too few.
  // For results in 16 bits the reduced one, rounded to 32 bits, goes to the hardware's sine and cosine, which take turns: 1.8e-7 off at
  // most with that rounding (over a million angles), a thousandth of what the result's own rounding is.  (The library's, at four times the
  // instructions: the 1M-token shard's rows, forward and backward, 57.6 -> 60.4 us, prompts appended in half 8.9 -> 10.4.)
  // Results in 32 bits would show it.  They get the library's, and to first order what the rounding of the reduced angle left out.
  __device__ __forceinline__ void turn(const RopeRow& r, int s, int64_t pos) {
    const double p = (double)pos * 0.15915494309189535;   // 1 / (2 pi)
#pragma unroll
    for (int i = 0; i < V; i += 4) {
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (turns) f = *reinterpret_cast<const float4*>(r.inv_freq + s * V + i);
      turn_one(p, f.x, i); turn_one(p, f.y, i + 1); turn_one(p, f.z, i + 2); turn_one(p, f.w, i + 3);
    }
  }
  __device__ __forceinline__ void turn_one(double p, float f, int i) {
    const double turns = p * (double)f;
    const double part = turns - __builtin_rint(turns);
    const float x = (float)part;
    if constexpr (std::is_same<E, float>::value) {
      float u, v;
      sincospif(2.f * x, &u, &v);
      const float left = 6.2831853f /* 2 pi */ * (float)(part - (double)x);
      sn[i] = fmaf(left, v, u);
      cs[i] = fmaf(-left, u, v);
    } else {
      sn[i] = __builtin_amdgcn_sinf(x);
      cs[i] = __builtin_amdgcn_cosf(x);
    }
  }

  // the lane's 2 V weights (ones if there are none)
  __device__ __forceinline__ void weights(const float* w, float (&out)[2 * V]) const {
#pragma unroll
    for (int i = 0; i < 2 * V; i += 4) {
      const float4 x = w ? *reinterpret_cast<const float4*>(w + (i < V ? a + i : b + i - V)) : make_float4(1.f, 1.f, 1.f, 1.f);
      out[i] = x.x; out[i + 1] = x.y; out[i + 2] = x.z; out[i + 3] = x.w;
    }
  }

  // pair i of the lane's elements
  static constexpr int first(int i) { return INTER ? 2 * i : i; }
  static constexpr int second(int i) { return INTER ? 2 * i + 1 : V + i; }

  __device__ __forceinline__ void rotate(float (&x)[2 * V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float u = x[first(i)], v = x[second(i)];
      x[first(i)] = turns ? u * cs[i] - v * sn[i] : u;
      x[second(i)] = turns ? u * sn[i] + v * cs[i] : v;
    }
  }
  __device__ __forceinline__ void rotate_back(float (&x)[2 * V]) const {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float u = x[first(i)], v = x[second(i)];
      x[first(i)] = turns ? u * cs[i] + v * sn[i] : u;
      x[second(i)] = turns ? v * cs[i] - u * sn[i] : v;
    }
  }

  // sum over the lanes of a row
  __device__ __forceinline__ float row_sum(const RopeRow& r, float x) const {
    x = holds ? x : 0.f;
    for (int m = 1 << r.lg >> 1; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
    return x;
  }
  __device__ __forceinline__ void row_sums(const RopeRow& r, float& x, float& y) const {
    x = holds ? x : 0.f;
    y = holds ? y : 0.f;
    for (int m = 1 << r.lg >> 1; m >= 1; m >>= 1) {
      x += __shfl_xor(x, m, 64);
      y += __shfl_xor(y, m, 64);
    }
  }
  __device__ __forceinline__ float rms(const RopeRow& r, const float (&x)[2 * V]) const {
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) sq += x[i] * x[i];
    return rsqrtf(row_sum(r, sq) * r.inv_d + r.eps);
  }

  // one row, as it is stored
  __device__ __forceinline__ void forward(const RopeRow& r, const float (&w)[2 * V], uint4& pa, uint4& pb) const {
    float x[2 * V];
    unpack16<E>(pa, x);
    unpack16<E>(pb, x + V);
    if (r.norm) {
      const float inv = rms(r, x);
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) x[i] = x[i] * inv * w[i];
    }
    rotate(x);
    pa = pack16<E>(x);
    pb = pack16<E>(x + V);
  }
};

template <class E>
struct StorageOf { typedef uint16_t type; };
template <>
struct StorageOf<float> { typedef float type; };

// Host side: the row geometry of a head (V elements in 16 bytes).
inline RopeRow make_rope_row(int head_dim, int rot_dim, int v, bool norm, float eps, const float* inv_freq) {
  RopeRow r{};
  r.pieces2 = head_dim / (2 * v);
  r.rot2 = rot_dim / (2 * v);
  while ((1 << r.lg) < r.pieces2) ++r.lg;
  r.norm = norm; r.eps = eps; r.inv_d = 1.f / (float)head_dim; r.inv_freq = inv_freq;
  return r;
}

}  // namespace loong
