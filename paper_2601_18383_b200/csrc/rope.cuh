// Rotary positions with one or several axes (time, height, width) on the queries and keys of a batch
// of tokens.  Pair i of a head's first `rot` columns turns by the angle
//     phi_i = pos[axis(i)] * theta^(-2 i / rot),      (a, b) -> (a cos phi - b sin phi, a sin phi + b cos phi)
// Bound by the bytes of q and k, each read and written once in 16-byte pieces (where sizes and strides are
// multiples of 16 bytes; element by element otherwise): a CTA computes the cosines and sines of its tokens
// once, in shared memory, and applies them to all heads.  16384 tokens of 32 + 8 heads of 128 in bf16: 59 us, 5.7 TB/s
// (0.87 of a copy).  The angle
// is formed in 64 bits as a number of revolutions and reduced before it is rounded to 32: at a
// position of a million an fp32 product would be off by 0.06 rad.
#pragma once

#include "common.cuh"

namespace dynts {

constexpr int kRopeMaxAxes = 4;
constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;       // tokens per CTA of a large batch
constexpr int kRopeMaxHalf = 128;    // pairs (head_dim <= 256)

struct RopeParams {
  const void* q;
  const void* k;   // or NULL
  void* q_out;
  void* k_out;
  long long q_stride, k_stride, qo_stride, ko_stride;  // elements between tokens
  const int* pos;  // [axes][n_tokens]
  int n_tokens, Hq, Hkv, d, rot, axes;
  int adjacent;    // pairs (2 i, 2 i + 1) instead of (i, i + rot / 2)
  int round_robin; // axes dealt out pair by pair instead of in blocks
  int section[kRopeMaxAxes];
  int tokens_per_cta;
  double log2_theta;
};

// The axis pair i takes its position from.
__device__ __forceinline__ int rope_axis(const RopeParams& p, int i) {
  if (!p.round_robin) {
    int a = 0;
    while (a < p.axes - 1 && i >= p.section[a]) i -= p.section[a++];
    return a;
  }
  // pairs are dealt to the axes in turn; an axis whose section is full is passed over
  int lvl = 0;  // whole rounds dealt so far
  for (;;) {
    int open = 0, next = 1 << 30;
#pragma unroll
    for (int a = 0; a < kRopeMaxAxes; ++a)
      if (a < p.axes && p.section[a] > lvl) {
        ++open;
        next = min(next, p.section[a]);
      }
    if (open == 0) return 0;
    if (i < (next - lvl) * open) {
      int x = i % open;
      for (int a = 0; a < p.axes; ++a)
        if (p.section[a] > lvl && x-- == 0) return a;
      return 0;
    }
    i -= (next - lvl) * open;
    lvl = next;
  }
}

template <typename T, int V>  // V elements at a time: 16 bytes, else one after another (no alignment is asked of them)
struct RopeVec {
  T x[V];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (V * sizeof(T) == 16) {
      *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) x[e] = p[e];
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (V * sizeof(T) == 16) {
      *reinterpret_cast<uint4*>(p) = *reinterpret_cast<const uint4*>(x);
    } else {
#pragma unroll
      for (int e = 0; e < V; ++e) p[e] = x[e];
    }
  }
};

template <typename T, int V>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(const __grid_constant__ RopeParams p) {
  __shared__ float2 cs[kRopeTokens * kRopeMaxHalf];
  const int half = p.rot >> 1;
  const int t0 = blockIdx.x * p.tokens_per_cta, nt = min(p.tokens_per_cta, p.n_tokens - t0);
  for (int x = threadIdx.x; x < nt * half; x += kRopeThreads) {
    const int t = x / half, i = x - t * half;
    // theta^(-2 i / rot) / (2 pi): revolutions per position
    const double f = exp2(-(double)i / (double)half * p.log2_theta) * 0.15915494309189535;
    const double turns = (double)p.pos[(size_t)rope_axis(p, i) * p.n_tokens + t0 + t] * f;
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[t * half + i] = make_float2(c, s);
  }
  __syncthreads();
  const int turn_units = p.adjacent ? p.rot / V : half / V;  // a unit: V pairs of halves, or V / 2 adjacent pairs
  const int units = turn_units + (p.d - p.rot) / V;          // the columns behind `rot` pass through
  const int heads = p.Hq + (p.k ? p.Hkv : 0);
  const int work = nt * heads * units;
#pragma unroll 2
  for (int w = threadIdx.x; w < work; w += kRopeThreads) {
    const int u = w % units, th = w / units, head = th % heads, t = th / heads;
    const bool isq = head < p.Hq;
    const T* src = isq ? static_cast<const T*>(p.q) + (size_t)(t0 + t) * p.q_stride + (size_t)head * p.d
                       : static_cast<const T*>(p.k) + (size_t)(t0 + t) * p.k_stride + (size_t)(head - p.Hq) * p.d;
    T* dst = isq ? static_cast<T*>(p.q_out) + (size_t)(t0 + t) * p.qo_stride + (size_t)head * p.d
                 : static_cast<T*>(p.k_out) + (size_t)(t0 + t) * p.ko_stride + (size_t)(head - p.Hq) * p.d;
    RopeVec<T, V> a;
    if (u >= turn_units) {
      const int col = p.rot + (u - turn_units) * V;
      if (src == dst) continue;
      a.load(src + col);
      a.store(dst + col);
    } else if (p.adjacent) {
      if constexpr (V >= 2) {
        a.load(src + u * V);
        RopeVec<T, V> y;
#pragma unroll
        for (int e = 0; e < V; e += 2) {
          const float2 r = cs[t * half + u * (V / 2) + e / 2];
          const float x0 = to_float(a.x[e]), x1 = to_float(a.x[e + 1]);
          from_float(&y.x[e], x0 * r.x - x1 * r.y);
          from_float(&y.x[e + 1], x0 * r.y + x1 * r.x);
        }
        y.store(dst + u * V);
      }
    } else {
      RopeVec<T, V> b, ya, yb;
      a.load(src + u * V);
      b.load(src + half + u * V);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float2 r = cs[t * half + u * V + e];
        const float x0 = to_float(a.x[e]), x1 = to_float(b.x[e]);
        from_float(&ya.x[e], x0 * r.x - x1 * r.y);
        from_float(&yb.x[e], x0 * r.y + x1 * r.x);
      }
      ya.store(dst + u * V);
      yb.store(dst + half + u * V);
    }
  }
}

}  // namespace dynts
