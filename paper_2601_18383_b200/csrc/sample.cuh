// A token per row of logits x, from a given random number u in [0, 1).
//
//   w_i = exp((x_i - max x) / T)
// The tokens are ranked by x, equal ones by the lower index.  Kept are the first top_k of them; of those the shortest run
// from the first on whose weights add up to top_p of all of theirs; of those the ones with w >= min_p.  The token is the
// first in the order of the vocabulary at which the running sum of the kept weights exceeds u times their sum.
// T <= 0: the first maximum.
//
// The answer is a whole number, so what decides it is computed nearly exactly: weights in 64 bits to 2^-46, held as whole numbers
// of 2^-45, whose sums are the same in every order (vocabularies below 2^19).  A sum over 128256 of them is within 2^-28 of the
// exact one in the worst case and about 2^-38 in the mean, while an fp32 sum would move a border in one row of ten.
//
// A cluster of CTAs takes a row, every warp a run of it.  Every cut keeps a prefix of the ranking, so a row's cuts come down to
// one border, a (value, index) pair.  The first reading takes every lane's maximum; what follows depends on the row's settings:
//   * top_k up to 1024: a lane keeps the maxima of up to 16 groups of its vectors.  With c a value that q of a CTA's groups' maxima reach (the edge of a
//     step of a histogram of theirs), q tokens or more of the CTA lie at or above it; with q = top_k / CTAs and the smallest c of the
//     cluster's, top_k tokens or more do.  The tokens from there on are collected in a second reading of the groups that reach
//     it, a list per warp and so in order; the first CTA merges the lists, ranks them, and decides alone.
//   * top_p alone, a larger top_k, or lists that overflowed: a histogram over up to 1024 steps, of the tokens by the distance to the maximum, of the
//     weights by the 32nd part of a binary order; a second reading of the step in which the border lies, and the first CTA
//     ranks that.  Steps of many equal logits that overflow the lists are narrowed down by the bits of the value instead, and a
//     border inside equal values is a count of them.
//   * nothing cut off, or by min_p alone: no border is needed.
// Where the kept tokens are not in a list, the warps add up theirs, exchange the sums, and the CTA in which the token lies looks
// for it: sixteenths of the one warp's run, then the run of one warp.
//
// Bound by the bytes of the logits for many rows (and by the exponentials where all weights are added up), by the
// chain of readings and exchanges for few.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "evict.cuh"  // the cluster barrier

namespace dynts {

constexpr int kSmThreads = 512;
constexpr int kSmWarps = kSmThreads / 32;
constexpr int kSmWarpList = 128;     // tokens a warp can collect
constexpr int kSmList = 2048;        // tokens the first CTA can merge
constexpr int kSmMaxCluster = 8;
constexpr int kSmListK = 1024;       // top_k that lists are tried with
constexpr int kSmBins = 2 * kSmThreads;  // steps of a histogram
constexpr int kSmTable = 16;
constexpr int kSmGroups = 16;       // of a lane's vectors, whose maxima are kept
constexpr int kSmPerSm = 2;         // CTAs
constexpr double kSmFar = 33.0;      // of a token that weighs nothing, in units of T (32, and one for roundings)
constexpr int kSmNoStep = 1 << 20;   // of a token that weighs nothing
constexpr int kSmMaxVocab = (1 << 19) - 1;  // sums of 2^45 for each token fit 64 bits

struct SampleParams {
  const void* logits;
  long long row_stride;
  const float* u;
  const float* temperatures;  // [rows], or NULL: the scalars
  const int* top_ks;
  const float* top_ps;
  const float* min_ps;
  int* tokens;
  float* logprobs;  // or NULL
  int vocab, cluster;
  float temperature, top_p, min_p;
  int top_k;
};

typedef unsigned long long u64;

// Kept are the values above x and those equal to it up to `index`.
struct SmBorder {
  float x;
  int index;
  __device__ __forceinline__ bool keeps(float y, int i) const { return y > x || (y == x && i <= index); }
};

struct SmShared {
  double table[kSmTable]; // 2^(j / 16): a bank each for the lanes' lookups
  float warp_max[kSmWarps], warp_min[kSmWarps];
  u64 scan[kSmWarps];
  unsigned group_max[kSmGroups][kSmThreads];  // a word of maxima of each lane's groups
  // what the other CTAs of the cluster read
  float max, cut, low;    // largest logit; a value that enough tokens reach; smallest of the lanes' maxima
  unsigned lanes;         // that hold any
  unsigned warp_count[kSmWarps];
  unsigned warp_ties[kSmWarps];
  u64 warp_sum[kSmWarps];
  u64 outside;
  int verdict;            // of the first CTA: 1 decided, 0 a list overflowed
  int tie_index;
  SmBorder border;
  alignas(8) unsigned hist[2][kSmBins];  // low and high halves of 64-bit sums
  unsigned radix_count[256];
  unsigned radix_weight[2][256];
  uint2 list[kSmWarps][kSmWarpList];  // key, index
  // the rest is a CTA's own
  unsigned offset[kSmMaxCluster * kSmWarps + 1];
  int bin, digit;
  u64 above, below;
  double goal;
  unsigned count;
  u64 merged_weight[256];
  unsigned merged_count[256];
  u64 sort[kSmThreads];
  unsigned picked, key_min, key_max;
  int found;
  unsigned pick[kSmList];
  unsigned key[kSmList];  // the merged lists
  int index[kSmList];
  u64 weight[kSmList];
};

__device__ __forceinline__ void sm_cluster_sync(int cluster) {  // (also of shared memory within the CTA)
  if (cluster > 1) {
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
}

template <typename T>
__device__ __forceinline__ T sm_peer(const T* mine, int rank) {  // the same variable of another CTA of the cluster
  uint32_t at;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
  T x;
  if constexpr (sizeof(T) == 8) {
    u64 v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(at) : "memory");
    memcpy(&x, &v, 8);
  } else {
    unsigned v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    memcpy(&x, &v, 4);
  }
  return x;
}

// Adds to a 64-bit sum in shared memory as two 32-bit words: the sum of the low words wraps around in exactly one of the
// additions that carry.  (2.5 cycles per word and warp; one 64-bit addition is a loop of compare-and-swap, 19 to 57.)
template <int N>
__device__ __forceinline__ void sm_add(unsigned (&sum)[2][N], int at, u64 x) {
  const unsigned lo = (unsigned)x, old = atomicAdd(&sum[0][at], lo), hi = (unsigned)(x >> 32) + (old + lo < lo ? 1u : 0u);
  if (hi) atomicAdd(&sum[1][at], hi);
}

__device__ __forceinline__ unsigned sm_key(float x) {  // order-preserving; -0 and +0 alike
  const unsigned b = __float_as_uint(x + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float sm_value(unsigned key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }

// A row's weights exp((x - M) / T) in units of 2^-45.  With y = (x - M) / T: e^y = 2^(n / 16) e^f, n whole and |f| <= ln 2 / 32; the
// series of e^f to f^6 is off by less than 5e-16 of it.  Twelve operations in 64 bits: with the rest of a token's 25 instructions they
// bound the rows whose weights are all added up.  (64 table entries and a series to f^4: bank conflicts cost more than two operations.)
struct SmWeights {
  double top, inv_t;
  const double* table;
  static __device__ __forceinline__ int fine(int n, double f) { return -2 * n + ((unsigned)__double2hiint(f) > 0x80000000u ? 1 : 0); }  // (-0 is no less than 0)
  __device__ __forceinline__ int step(float x) const {
    const double y = ((double)x - top) * inv_t, magic = 6755399441055744.0, t = fma(y, 23.083120654223414, magic);
    if ((unsigned)__double2hiint(y) >= 0xc0400000u) return kSmNoStep;
    return fine(__double2loint(t), fma(t - magic, -0.04332169878499658, y));
  }
  __device__ __forceinline__ u64 operator()(float x) const {
    int n;
    return with_step(x, n);
  }
  // n: its step, 32 to a binary order down from 1 (below 2^-46: kSmNoStep); it never grows with x.
  __device__ __forceinline__ u64 with_step(float x, int& n) const {
    const double y = ((double)x - top) * inv_t;  // (the difference first: a largest logit of any size leaves its precision alone)
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the whole part
    const double t = fma(y, 23.083120654223414, magic);  // 16 / ln 2
    n = __double2loint(t);
    const double f = fma(t - magic, -0.04332169878499658, y);  // ln 2 / 16
    double e = fma(fma(fma(fma(fma(fma(1.0 / 720.0, f, 1.0 / 120.0), f, 1.0 / 24.0), f, 1.0 / 6.0), f, 0.5), f, 1.0), f, 1.0);
    const double g = table[n & (kSmTable - 1)];
    e = fma(__hiloint2double(__double2hiint(g) + (n >> 4) * (1 << 20), __double2loint(g)), e, 128.0);
    const u64 w = (u64)__double_as_longlong(e) - 0x4060000000000000ull;  // (128, whose mantissa's unit is 2^-45)
    const bool some = (unsigned)__double2hiint(y) < 0xc0400000u;  // (y <= -32: less than half a unit.  No branch: several tokens' chains side by side)
    n = some ? fine(n, f) : kSmNoStep;
    return some ? w : 0ull;
  }
};

__device__ __forceinline__ float sm_max_nan(float a, float b) {  // a NaN stays
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ unsigned sm_max2_nan(unsigned a, unsigned b) {  // of two bf16 each
  unsigned y;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}

// A vector that begins at element i of the row and is not all within it.
template <typename X>
__device__ __noinline__ uint4 sm_edge(const X* at, int i, int vocab) {
  constexpr int E = 16 / (int)sizeof(X);
  unsigned w[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    if constexpr (E == 4) {
      w[q] = i + q >= 0 && i + q < vocab ? __float_as_uint(at[q]) : 0xff800000u;
    } else {
      w[q] = 0xff80ff80u;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int e = 2 * q + h;
        if (i + e >= 0 && i + e < vocab) w[q] = (w[q] & (h ? 0x0000ffffu : 0xffff0000u)) | ((unsigned)__bfloat16_as_ushort(at[e]) << (16 * h));
      }
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// A row in 16-byte vectors, from the boundary at or before its first element; what lies outside the row reads as -inf, which
// weighs nothing.
template <typename X>
struct SmRow {
  static constexpr int E = 16 / (int)sizeof(X);
  const X* base;   // aligned down to 16 bytes
  int skew;        // elements between there and the row
  int vocab;
  int v0, v1;      // this warp's vectors
  int rounds;      // of 128 vectors of a warp, in a group
  __device__ __forceinline__ uint4 load(int v) const {
    const int i = v * E - skew;
    if (i >= 0 && i + E <= vocab) return *reinterpret_cast<const uint4*>(base + (size_t)v * E);
    return sm_edge(base + (size_t)v * E, i, vocab);
  }
  static __device__ __forceinline__ float at(const uint4& w, int e) {
    const unsigned q[4] = {w.x, w.y, w.z, w.w};
    if constexpr (E == 4) return __uint_as_float(q[e]);
    else return __uint_as_float((e & 1) ? q[e >> 1] & 0xffff0000u : q[e >> 1] << 16);
  }
  // Running maxima, a word: of floats, or of two bf16 (a NaN stays).
  static __device__ __forceinline__ unsigned start() { return E == 4 ? 0xff800000u : 0xff80ff80u; }
  static __device__ __forceinline__ unsigned more(unsigned m, const uint4& w) {
    if constexpr (E == 4)
      return __float_as_uint(sm_max_nan(sm_max_nan(sm_max_nan(__uint_as_float(m), __uint_as_float(w.x)), sm_max_nan(__uint_as_float(w.y), __uint_as_float(w.z))), __uint_as_float(w.w)));
    else return sm_max2_nan(sm_max2_nan(m, sm_max2_nan(w.x, w.y)), sm_max2_nan(w.z, w.w));
  }
  static __device__ __forceinline__ float largest(unsigned m) {
    if constexpr (E == 4) return __uint_as_float(m);
    else return sm_max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
};

// This lane's vectors of a warp's run, four loads at a time.
template <typename X, typename F>
__device__ __forceinline__ void each_vector(const SmRow<X>& r, int v0, int v1, F f) {
  for (int v = v0 + (int)(threadIdx.x & 31); v < v1; v += 128) {
    uint4 w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (v + 32 * q < v1) w[q] = r.load(v + 32 * q);
#pragma unroll
    for (int q = 0; q < 4; ++q)
      if (v + 32 * q < v1) f(v + 32 * q, w[q]);
  }
}

template <typename V>
__device__ __forceinline__ V sm_warp_scan(V x) {  // inclusive
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  return x;
}
// The sum of what lies before, over the CTA's threads; every thread gets the total.
__device__ __forceinline__ u64 sm_scan(u64 x, u64* warps, u64& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const u64 s = sm_warp_scan(x);
  __syncthreads();
  if (lane == 31) warps[warp] = s;
  __syncthreads();
  u64 before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kSmWarps; ++w) {
    const u64 y = warps[w];
    if (w < warp) before += y;
    total += y;
  }
  return before + s - x;
}

// Whether a running sum passes its goal with this addend: the first one does, or it had not been reached before.
__device__ __forceinline__ bool sm_passes(u64 before, u64 here, double goal) {
  return here > 0 && (double)(before + here) >= goal && (before == 0 || (double)before < goal);
}

// By all threads of a CTA: the token of the merged list at which the running sum down the ranking passes its goal, `above` lying before
// them all: a histogram of the distance to `from` in steps, then the tokens of one step against one another.  Sums are of the weights or of
// the tokens that `outer` keeps.  -1: the sum does not get there.
__device__ __noinline__ int sm_pick(SmShared& sh, unsigned n, u64 above, double goal, bool by_weight, SmBorder outer, float from, float steps) {
  const int tid = threadIdx.x;
  auto amount = [&](unsigned i) { return outer.keeps(sm_value(sh.key[i]), sh.index[i]) ? by_weight ? sh.weight[i] : 1ull : 0ull; };
  auto step = [&](unsigned i) { return max(0, min(kSmBins - 1, (int)((from - sm_value(sh.key[i])) * steps))); };
  for (int q = 0; q < 2; ++q) sh.hist[0][tid + q * kSmThreads] = sh.hist[1][tid + q * kSmThreads] = 0;
  if (tid == 0) sh.digit = sh.found = -1, sh.picked = 0, sh.key_min = 0xffffffffu, sh.key_max = 0;
  __syncthreads();
  for (unsigned i = tid; i < n; i += kSmThreads) {
    const u64 a = amount(i);
    if (a) sm_add(sh.hist, step(i), a);
  }
  __syncthreads();
  u64 here[2], all;
#pragma unroll
  for (int q = 0; q < 2; ++q) here[q] = sh.hist[0][2 * tid + q] + ((u64)sh.hist[1][2 * tid + q] << 32);
  const u64 before = sm_scan(here[0] + here[1], sh.scan, all) + above;
  if (sm_passes(before, here[0] + here[1], goal)) {
    const bool second = !sm_passes(before, here[0], goal);
    sh.digit = 2 * tid + (second ? 1 : 0);
    sh.below = before + (second ? here[0] : 0ull);
  }
  __syncthreads();
  const int bin = sh.digit;
  if (bin >= 0) {
    for (unsigned i = tid; i < n; i += kSmThreads)
      if (step(i) == bin && amount(i)) {
        sh.pick[atomicAdd(&sh.picked, 1u)] = i;
        atomicMin(&sh.key_min, sh.key[i]);
        atomicMax(&sh.key_max, sh.key[i]);
      }
    __syncthreads();
    const unsigned m = sh.picked;
    if (m > 32 && sh.key_min == sh.key_max) {
      // equal values (logits of 16 bits): the list is in the order of the vocabulary, so its place is a count
      const u64 one = by_weight ? sh.weight[sh.pick[0]] : 1ull;
      const double need = ceil((goal - (double)sh.below) / (double)one);
      u64 t = need <= 1.0 ? 1ull : need >= (double)m ? (u64)m : (u64)need;
      while (t > 1 && (double)(sh.below + (t - 1) * one) >= goal) --t;
      while (t < m && (double)(sh.below + t * one) < goal) ++t;
      constexpr unsigned N = kSmList / kSmThreads;
      u64 mine = 0, ties;
      for (unsigned i = N * tid; i < min(n, N * (tid + 1)); ++i) mine += step(i) == bin && amount(i) ? 1ull : 0ull;
      u64 seen = sm_scan(mine, sh.scan, ties);
      for (unsigned i = N * tid; i < min(n, N * (tid + 1)); ++i)
        if (step(i) == bin && amount(i) && ++seen == t) sh.found = (int)i;
    } else for (unsigned e = tid; e < m; e += kSmThreads) {
      const unsigned i = sh.pick[e], key = sh.key[i];
      const int index = sh.index[i];
      u64 run = sh.below;
      for (unsigned o = 0; o < m; ++o) {
        const unsigned j = sh.pick[o], other = sh.key[j];
        if (other > key || (other == key && sh.index[j] < index)) run += by_weight ? sh.weight[j] : 1ull;
      }
      if (sm_passes(run, by_weight ? sh.weight[i] : 1ull, goal)) sh.found = (int)i;
    }
    __syncthreads();
  }
  const int found = sh.found;
  __syncthreads();
  for (int q = 0; q < 2; ++q) sh.hist[0][tid + q * kSmThreads] = sh.hist[1][tid + q * kSmThreads] = 0;
  __syncthreads();
  return found;
}

// (64 registers for two CTAs per SM, with 224 bytes of spill stores: the ways to a border are many, and a row walks through one or two.)
template <typename X>
__global__ void __launch_bounds__(kSmThreads, kSmPerSm) sample_kernel(const __grid_constant__ SampleParams p) {
  constexpr int E = SmRow<X>::E;
  extern __shared__ __align__(16) uint8_t sm_raw[];
  SmShared& sh = *reinterpret_cast<SmShared*>(sm_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cluster = p.cluster, row = (int)blockIdx.x / cluster, rank = (int)blockIdx.x - row * cluster;
  const int lists = cluster * kSmWarps;

  SmRow<X> r;
  {
    const X* x0 = static_cast<const X*>(p.logits) + (size_t)row * p.row_stride;
    r.skew = (int)((reinterpret_cast<uintptr_t>(x0) & 15u) / sizeof(X));
    r.base = x0 - r.skew;
    r.vocab = p.vocab;
    const int vectors = (r.skew + p.vocab + E - 1) / E, per = (vectors + cluster - 1) / cluster;
    const int c0 = min(vectors, rank * per), c1 = min(vectors, c0 + per), mine = (c1 - c0 + kSmWarps - 1) / kSmWarps;
    r.v0 = min(c1, c0 + warp * mine);
    r.v1 = min(c1, r.v0 + mine);
    r.rounds = max(1, (mine + 128 * kSmGroups - 1) / (128 * kSmGroups));  // (the same in every warp)
  }
  // the row's settings
  float T = p.temperatures ? p.temperatures[row] : p.temperature, top_p = p.top_ps ? p.top_ps[row] : p.top_p;
  float min_p = p.min_ps ? p.min_ps[row] : p.min_p, u = p.u[row];
  int top_k = p.top_ks ? p.top_ks[row] : p.top_k;
  u = u >= 1.f ? 0.99999994f : u >= 0.f ? u : 0.f;
  if (!(T > 0.f)) T = 1.f, top_k = 1, u = 0.f;
  if (top_k <= 0 || top_k >= p.vocab) top_k = 0;
  if (top_k == 1 || !(top_p < 1.f)) top_p = 1.f;
  top_p = fmaxf(top_p, 0.f);
  const bool cut_p = top_p < 1.f;
  T = fminf(T, 3.402823466e38f);
  const double inv_t = 1.0 / (double)T;
  const int share = (top_k + cluster - 1) / cluster;  // of top_k, for each CTA
  const bool listed = top_k > 0 && top_k <= kSmListK;

  // ---- every lane's maximum
  float top;
  {
    unsigned m = SmRow<X>::start();
    unsigned mg = SmRow<X>::start();
    int g = 0, left = r.rounds;
    for (int v = r.v0 + lane; v < r.v1; v += 128) {
      uint4 w[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (v + 32 * q < r.v1) w[q] = r.load(v + 32 * q);
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (v + 32 * q < r.v1) mg = SmRow<X>::more(mg, w[q]);
      if (--left == 0 || v + 128 >= r.v1) {
        sh.group_max[g++][tid] = mg;
        m = SmRow<X>::more(m, make_uint4(mg, mg, mg, mg));
        mg = SmRow<X>::start();
        left = r.rounds;
      }
    }
    top = SmRow<X>::largest(m);
  }
  if (tid < kSmTable) sh.table[tid] = exp2((double)tid / kSmTable);
  for (int q = 0; q < 2; ++q) sh.hist[0][tid + q * kSmThreads] = sh.hist[1][tid + q * kSmThreads] = 0;
  const float lane_top = top;
  float least = top > -INFINITY ? top : INFINITY;  // of the lanes that hold anything
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    top = sm_max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
  }
  if (lane == 0) sh.warp_max[warp] = top, sh.warp_min[warp] = least;
  const unsigned lanes = (unsigned)__syncthreads_count(lane_top > -INFINITY);
#pragma unroll
  for (int w = 0; w < kSmWarps; ++w) top = sm_max_nan(top, sh.warp_max[w]), least = fminf(least, sh.warp_min[w]);
  float cut = -INFINITY;
  if (listed && share == 1) {
    cut = top;
  } else if (listed) {
    // a value that `share` of the groups' maxima reach, close to the largest such: by a histogram of 512 equal steps
    least = fmaxf(least, __double2float_rd((double)top - kSmFar * (double)T));
    const float steps = top > least ? (kSmThreads - 1) / (top - least) : 0.f;
    const int mine = r.v0 + lane < r.v1 ? (r.v1 - r.v0 - lane + 128 * r.rounds - 1) / (128 * r.rounds) : 0;  // this lane's groups
    auto step_of = [&](float x) { return x > -INFINITY ? min(kSmThreads - 1, max(0, (int)((top - x) * steps))) : kSmThreads; };
    for (int g = 0; g < mine; ++g) {
      const int b = step_of(SmRow<X>::largest(sh.group_max[g][tid]));  // (those below the lanes' maxima: the last step)
      if (b < kSmThreads) atomicAdd(&sh.hist[0][b], 1u);
    }
    u64 all;
    if (tid == 0) sh.bin = kSmThreads;
    const u64 before = (__syncthreads(), sm_scan(sh.hist[0][tid], sh.scan, all)), here = sh.hist[0][tid];
    if (before < (u64)share && before + here >= (u64)share) sh.bin = tid;
    __syncthreads();
    if (sh.bin < kSmThreads) {  // (fewer groups hold anything: all is collected)
      float reach = INFINITY;
      for (int g = 0; g < mine; ++g) {
        const float x = SmRow<X>::largest(sh.group_max[g][tid]);
        if (step_of(x) <= sh.bin) reach = fminf(reach, x);
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) reach = fminf(reach, __shfl_xor_sync(0xffffffffu, reach, o));
      if (lane == 0) sh.warp_min[warp] = reach;
      __syncthreads();
      cut = INFINITY;
#pragma unroll
      for (int w = 0; w < kSmWarps; ++w) cut = fminf(cut, sh.warp_min[w]);
    }
    sh.hist[0][tid] = 0;
  }
  if (tid == 0) sh.max = top, sh.cut = cut, sh.low = least, sh.lanes = lanes;
  sm_cluster_sync(cluster);
  float M, low_all;
  unsigned lanes_all = 0;
  {
    float a = -INFINITY, b = INFINITY, c = INFINITY;
    if (lane < cluster) a = sm_peer(&sh.max, lane), b = sm_peer(&sh.cut, lane), c = sm_peer(&sh.low, lane), lanes_all = sm_peer(&sh.lanes, lane);
    lanes_all = __reduce_add_sync(0xffffffffu, lanes_all);
#pragma unroll
    for (int o = kSmMaxCluster / 2; o > 0; o >>= 1) {
      a = sm_max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
      b = fminf(b, __shfl_xor_sync(0xffffffffu, b, o));
      c = fminf(c, __shfl_xor_sync(0xffffffffu, c, o));
    }
    M = __shfl_sync(0xffffffffu, a, 0);
    cut = __shfl_sync(0xffffffffu, b, 0);
    low_all = __shfl_sync(0xffffffffu, c, 0);
  }
  const double Md = (double)M;
  // what min_p keeps: x >= least_x (min_p > 1 counts as 1)
  const float least_x = min_p > 0.f ? __double2float_ru(fmin(Md + (double)T * log((double)min_p), Md)) : -INFINITY;
  // Below this a token weighs nothing, and what is counted, collected or kept of such tokens changes no answer: distances end here, so
  // that logits of the type's lowest value (a usual mask) do not make steps of 3e35.
  const float far_x = __double2float_rd(Md - kSmFar * (double)T);
  cut = fmaxf(cut, far_x);
  low_all = fmaxf(low_all, far_x);
  const SmWeights weight_of{Md, inv_t, sh.table};
  auto answer = [&](int token, float x, u64 total) {
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = (float)(((double)x - Md) * inv_t - log((double)total * 2.842170943040401e-14));  // 2^-45
  };
  // The tokens for which wanted(x, index) holds, of those from `reach` up to `from`: a list per warp.  `deep`: most vectors reach that far, and few
  // of their elements lie in the range (a CTA's cycles, 60 rows of bf16: 3000 -> 2650, 64 of fp32: 21900 -> 21000; lists of
  // the largest are slower so: 800 rows 113 -> 117 us).
  auto collect = [&](float reach, float from, auto deep, auto wanted) {
    if (lane == 0) sh.warp_count[warp] = 0;
    __syncwarp();
    const int step = 128 * r.rounds;
    unsigned hits = 0;  // a bit for each of the lane's groups
#pragma unroll
    for (int g = 0; g < kSmGroups; ++g)
      if (r.v0 + lane + g * step < r.v1 && SmRow<X>::largest(sh.group_max[g][tid]) >= reach) hits |= 1u << g;
    for (; hits; hits &= hits - 1) {
      const int g0 = r.v0 + lane + (__ffs(hits) - 1) * step, g1 = min(r.v1, g0 + step);
      for (int v = g0; v < g1; v += 128) {
        uint4 ws[4];
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (v + 32 * q < g1) ws[q] = r.load(v + 32 * q);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          if (v + 32 * q >= g1 || !(SmRow<X>::largest(SmRow<X>::more(SmRow<X>::start(), ws[q])) >= reach)) continue;
          auto take = [&](float x, int i) {
            if (x > -INFINITY && wanted(x, i)) {
              const unsigned at = atomicAdd(&sh.warp_count[warp], 1u);
              if (at < kSmWarpList) sh.list[warp][at] = make_uint2(sm_key(x), (unsigned)i);
            }
          };
          if constexpr (decltype(deep)::value) {
            unsigned some = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float x = SmRow<X>::at(ws[q], e);
              some |= (x >= reach && x <= from ? 1u : 0u) << e;
            }
            for (; some; some &= some - 1) {
              const int e = __ffs(some) - 1, at_word = E == 4 ? e : e >> 1;
              const unsigned word = at_word < 2 ? (at_word == 0 ? ws[q].x : ws[q].y) : at_word == 2 ? ws[q].z : ws[q].w;
              take(__uint_as_float(E == 4 ? word : (e & 1) ? word & 0xffff0000u : word << 16), (v + 32 * q) * E + e - r.skew);
            }
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) take(SmRow<X>::at(ws[q], e), (v + 32 * q) * E + e - r.skew);
          }
        }
      }
    }
    __syncwarp();
    // in the order of the vocabulary: each token's place is the count of those before it
    const unsigned count = min(sh.warp_count[warp], (unsigned)kSmWarpList);
    uint2 mine[kSmWarpList / 32];
    unsigned place[kSmWarpList / 32];
#pragma unroll
    for (int q = 0; q < kSmWarpList / 32; ++q) {
      place[q] = 0;
      if (32 * q + lane < count) mine[q] = sh.list[warp][32 * q + lane];
    }
    for (unsigned j = 0; j < count; ++j) {
      const unsigned other = sh.list[warp][j].y;
#pragma unroll
      for (int q = 0; q < kSmWarpList / 32; ++q)
        if (32 * q + lane < count && other < mine[q].y) ++place[q];
    }
    __syncwarp();
#pragma unroll
    for (int q = 0; q < kSmWarpList / 32; ++q)
      if (32 * q + lane < count) sh.list[warp][place[q]] = mine[q];
  };
  // By the first CTA, behind a barrier: the lists as one, in order, with their weights.  How many; more than kSmList: overflowed.
  auto merge = [&]() -> unsigned {
    __syncthreads();
    if (warp == 0) {
      constexpr int N = kSmMaxCluster * kSmWarps / 32;  // neighbouring lists per lane
      unsigned c[N], sum = 0, most = 0;
#pragma unroll
      for (int q = 0; q < N; ++q) c[q] = lane * N + q < lists ? sm_peer(&sh.warp_count[(lane * N + q) % kSmWarps], (lane * N + q) / kSmWarps) : 0u;
#pragma unroll
      for (int q = 0; q < N; ++q) sum += c[q], most = max(most, c[q]);
      const unsigned upto = sm_warp_scan(sum);
      unsigned base = upto - sum;
#pragma unroll
      for (int q = 0; q < N; ++q) {
        sh.offset[lane * N + q] = base;
        base += c[q];
      }
      const bool over = __any_sync(0xffffffffu, most > kSmWarpList);
      if (lane == 31) sh.count = over ? kSmList + 1 : upto;
    }
    __syncthreads();
    const unsigned n = sh.count;
    if (n <= kSmList)
      for (unsigned i = tid; i < n; i += kSmThreads) {
        int lo = 0, hi = lists;  // the last list that begins at or before i (of equal ones the last, which holds it)
        while (hi - lo > 1) {
          const int mid = (lo + hi) >> 1;
          if (sh.offset[mid] <= i) lo = mid;
          else hi = mid;
        }
        const uint2 y = sm_peer(&sh.list[lo % kSmWarps][i - sh.offset[lo]], lo / kSmWarps);
        sh.key[i] = y.x;
        sh.index[i] = (int)y.y;
        sh.weight[i] = weight_of(sm_value(y.x));
      }
    __syncthreads();
    return n;
  };
  // By the first CTA: the border among the merged tokens: the first `want` are kept, of those the shortest run whose
  // weights reach part of theirs (part < 0: all), or reach `goal` with `above` before them (goal >= 0).  from: no token is above it.
  auto rank_list = [&](unsigned n, unsigned want, double part, u64 above, double goal, float from) -> SmBorder {
    if (n <= kSmThreads / 2) {
      // few: each token's rank and the weights before it by comparing it with all, several threads to a token
      int per = 2;
      while (per < 32 && per * 2 * n <= kSmThreads) per *= 2;
      const unsigned i = tid / per, j0 = tid % per;
      u64 mine = 0, run = 0, total = 0;
      unsigned place = 0;
      if (tid < n) sh.sort[tid] = ((u64)sh.key[tid] << 32) | (0xffffffffu - tid);
      if (tid == 0) sh.count = 0;
      __syncthreads();
      if (i < n) mine = sh.sort[i];
      for (unsigned j = j0; j < n; j += per) {
        const bool before = sh.sort[j] > mine;
        place += before ? 1u : 0u;
        run += before ? sh.weight[j] : 0ull;
      }
      for (int o = per / 2; o > 0; o >>= 1) place += __shfl_xor_sync(0xffffffffu, place, o), run += __shfl_xor_sync(0xffffffffu, run, o);
      const bool counts = i < n && place < want;
      if (counts && j0 == 0 && place + 1 == min(n, want)) sh.below = run + sh.weight[i];  // of all that count
      __syncthreads();
      total = sh.below;
      const bool whole = goal < 0.0 && part < 0.0;
      const double reach = goal >= 0.0 ? goal : part * (double)total;
      const bool kept = counts && (whole || place + above == 0 || (double)(above + run) < reach);
      const unsigned most = __reduce_max_sync(0xffffffffu, kept ? place + 1 : 0u);
      if (lane == 0 && most > 0) atomicMax(&sh.count, most);
      __syncthreads();
      if (i < n && j0 == 0 && place + 1 == sh.count) sh.border = SmBorder{sm_value(sh.key[i]), sh.index[i]};
      __syncthreads();
      return sh.border;
    }
    float least = INFINITY;
    for (unsigned i = tid; i < n; i += kSmThreads) least = fminf(least, sm_value(sh.key[i]));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) least = fminf(least, __shfl_xor_sync(0xffffffffu, least, o));
    if (lane == 0) sh.warp_min[warp] = least;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSmWarps; ++w) least = fminf(least, sh.warp_min[w]);
    const float steps = from > least ? fminf((kSmBins - 1) / (from - least), 1e30f) : 0.f;
    SmBorder b{-INFINITY, -1};
    auto take = [&](int at) {
      if (at >= 0) b = SmBorder{sm_value(sh.key[at]), sh.index[at]};
    };
    if (goal >= 0.0) {
      take(sm_pick(sh, n, above, goal, true, b, from, steps));
    } else {
      take(sm_pick(sh, n, 0, (double)min(want, n), false, b, from, steps));
      if (part >= 0.0) {
        u64 mine = 0, all;
        for (unsigned i = tid; i < n; i += kSmThreads) mine += b.keeps(sm_value(sh.key[i]), sh.index[i]) ? sh.weight[i] : 0ull;
        sm_scan(mine, sh.scan, all);
        take(sm_pick(sh, n, 0, part * (double)all, true, b, from, steps));
      }
    }
    if (tid == 0) sh.border = b;
    __syncthreads();
    return b;
  };
  bool done = false;
  SmBorder border{-INFINITY, -1};
  if (!(M > -INFINITY && M < INFINITY)) {  // NaN or +inf somewhere, or nothing but -inf
    if (rank == 0 && tid == 0) {
      p.tokens[row] = -1;
      if (p.logprobs) p.logprobs[row] = NAN;
    }
    done = true;
  }
  if (!done && listed) {
    collect(cut, M, std::false_type{}, [&](float x, int) { return x >= cut; });
    sm_cluster_sync(cluster);
    if (rank == 0) {
      const unsigned n = merge();
      if (n <= kSmList) {
        const SmBorder b = rank_list(n, (unsigned)top_k, cut_p ? (double)top_p : -1.0, 0, -1.0, M);
        // the kept tokens' running sums, in the order of the vocabulary: neighbours per thread
        constexpr int N = kSmList / kSmThreads;
        u64 w[N], sum = 0, all;
#pragma unroll
        for (int q = 0; q < N; ++q) {
          const unsigned i = N * tid + q;
          w[q] = i < n && b.keeps(sm_value(sh.key[i]), sh.index[i]) && sm_value(sh.key[i]) >= least_x ? sh.weight[i] : 0ull;
          sum += w[q];
        }
        u64 run = sm_scan(sum, sh.scan, all);
        const u64 target = min((u64)__double2ull_rd((double)u * (double)all), all - 1);
        if (run <= target && run + sum > target) {
          unsigned i = N * tid;
#pragma unroll
          for (int q = 0; q < N - 1; ++q) {
            run += w[q];
            if (run <= target) i = N * tid + q + 1;
          }
          answer(sh.index[i], sm_value(sh.key[i]), all);
        }
      }
      if (tid == 0) sh.verdict = n <= kSmList ? 1 : 0;
    }
    sm_cluster_sync(cluster);
    done = sm_peer(&sh.verdict, 0) != 0;
  }
  if (!done) {
    // ---- the border by a histogram: first of the tokens (top_k), then of the weights of those kept (top_p)
    for (int which = 0; which < 2; ++which) {
      const bool by_weight = which == 1;
      if (by_weight ? !cut_p : top_k == 0) continue;
      // Weights: steps of a thirty-second of a binary order.  What lies beyond ln(V / (1 - p)) in units of T adds up to less than 1 - p of
      // the largest, so no border lies there and no step is counted.  Tokens: equal steps of the distance to the maximum up to `half`;
      // the lanes' maxima reach down to low_all; beyond their number, the smallest logit does.
      // (Distances are halved: two logits may be further apart than the largest number.)
      float half = 0.f;
      int bins = kSmBins, coarse = 0;  // (two steps as one where 1024 do not reach)
      if (by_weight) {
        bins = 2 + (int)(46.17f * (logf((float)p.vocab / (1.f - top_p)) + 0.01f));  // 32 / ln 2
        if (bins > kSmBins) coarse = 1, bins = kSmBins;
      } else if ((unsigned)top_k <= lanes_all) {
        half = 0.5f * M - 0.5f * low_all;
      } else {
        float least_all = INFINITY;
        each_vector(r, r.v0, r.v1, [&](int, const uint4& w) {
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float x = SmRow<X>::at(w, e);
            if (x > -INFINITY) least_all = fminf(least_all, x);
          }
        });
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) least_all = fminf(least_all, __shfl_xor_sync(0xffffffffu, least_all, o));
        __syncthreads();
        if (lane == 0) sh.warp_min[warp] = least_all;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kSmWarps; ++w) least_all = fminf(least_all, sh.warp_min[w]);
        if (tid == 0) sh.low = least_all;
        sm_cluster_sync(cluster);
        for (int k = 0; k < cluster; ++k) least_all = fminf(least_all, sm_peer(&sh.low, k));
        half = 0.5f * M - 0.5f * fmaxf(least_all, far_x);
      }
      const float steps = half > 0.f ? fminf((kSmBins - 1) / half, 1e30f) : 0.f;
      const float reach_all = M - half * 2.02f;  // (a step more than the span)
      auto bin_of = [&](float x) {  // (never grows with x: every rounding is monotone)
        if (by_weight) {
          const int n = weight_of.step(x) >> coarse;
          return n < bins ? n : kSmBins;
        }
        const float y = fmaf(x, -0.5f, 0.5f * M) * steps;
        return y < (float)kSmBins ? (int)y : kSmBins;
      };
      u64 outside = 0;
      each_vector(r, r.v0, r.v1, [&](int v, const uint4& w) {
        if (!by_weight && !(SmRow<X>::largest(SmRow<X>::more(SmRow<X>::start(), w)) >= reach_all)) return;
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float x = SmRow<X>::at(w, e);
          if (!border.keeps(x, v * E + e - r.skew)) continue;
          if (by_weight) {
            int b;
            const u64 w = weight_of.with_step(x, b);
            b >>= coarse;
            if (b < bins) sm_add(sh.hist, b, w);
            else outside += w;
          } else {
            const int b = bin_of(x);
            if (b < kSmBins) atomicAdd(&sh.hist[0][b], 1u);
          }
        }
      });
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) outside += __shfl_xor_sync(0xffffffffu, outside, o);
      __syncthreads();
      if (lane == 0) sh.scan[warp] = outside;
      __syncthreads();
      if (tid == 0) {
        u64 s = 0;
        for (int w = 0; w < kSmWarps; ++w) s += sh.scan[w];
        sh.outside = s;
        sh.bin = -1;
      }
      sm_cluster_sync(cluster);
      if (rank == 0) {
        u64 here[2] = {0, 0}, beyond = 0, all;
#pragma unroll 1
        for (int k0 = 0; k0 < cluster; k0 += 4) {  // (a CTA's two neighbouring steps in one word of 64 bits, low and high halves; counts have no high ones)
          u64 lo[4], hi[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            lo[k] = k0 + k < cluster ? sm_peer(reinterpret_cast<const u64*>(&sh.hist[0][2 * tid]), k0 + k) : 0ull;
            hi[k] = k0 + k < cluster ? sm_peer(reinterpret_cast<const u64*>(&sh.hist[1][2 * tid]), k0 + k) : 0ull;
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            here[0] += (lo[k] & 0xffffffffull) + (hi[k] << 32);
            here[1] += (lo[k] >> 32) + (hi[k] & 0xffffffff00000000ull);
          }
        }
        if (by_weight)
          for (int k = 0; k < cluster; ++k) beyond += sm_peer(&sh.outside, k);
        const u64 before = sm_scan(here[0] + here[1], sh.scan, all);
        const double g = by_weight ? (double)top_p * (double)(all + beyond) : (double)top_k;
        if (sm_passes(before, here[0] + here[1], g)) {
          const bool second = !sm_passes(before, here[0], g);
          sh.bin = 2 * tid + (second ? 1 : 0);
          sh.above = before + (second ? here[0] : 0ull);
          sh.goal = g;
        }
      }
      sm_cluster_sync(cluster);
      const int bin = sm_peer(&sh.bin, 0);
      const u64 above = sm_peer(&sh.above, 0);
      const double goal = sm_peer(&sh.goal, 0);
      for (int q = 0; q < 2; ++q) sh.hist[0][tid + q * kSmThreads] = sh.hist[1][tid + q * kSmThreads] = 0;
      if (bin < 0) {      // fewer tokens of any weight than top_k; or a sum missed by a rounding: all are kept
        __syncthreads();  // (the next histogram begins with cleared words)
        continue;
      }
      const SmBorder outer = border;
      // (a vector without an element of this bin or a nearer one is passed over: what the bin holds is at least this large)
      const float reach = by_weight ? __double2float_rd(Md - (double)(((bin + 1) << coarse) + 1) * 0.02166084939249829 * (double)T)  // ln 2 / 32
                          : steps > 0.f ? 2.f * (0.5f * M - (float)(bin + 2) / steps) : -INFINITY;
      const float from = by_weight ? fminf(M, __double2float_ru(Md - (double)((bin << coarse) - 2) * 0.02166084939249829 * (double)T)) : steps > 0.f ? fminf(M, 2.f * (0.5f * M - (float)(bin - 1) / steps)) : M;
      auto in_bin = [&](float x, int i) { return x >= reach && x <= from && bin_of(x) == bin && outer.keeps(x, i); };
      collect(reach, from, std::true_type{}, in_bin);
      sm_cluster_sync(cluster);
      if (rank == 0) {
        const unsigned n = merge();
        if (n <= kSmList) rank_list(n, by_weight ? n : (unsigned)((u64)top_k - above), -1.0, above, by_weight ? goal : -1.0, from);
        if (tid == 0) sh.verdict = n <= kSmList ? 1 : 0;
      }
      sm_cluster_sync(cluster);
      if (sm_peer(&sh.verdict, 0) != 0) {
        border.x = sm_peer(&sh.border.x, 0);
        border.index = sm_peer(&sh.border.index, 0);
        sm_cluster_sync(cluster);
        continue;
      }
      // ---- too many tokens of one step: by the bits of their keys, eight at a time
      unsigned lo = 0, at = 0;
      u64 over = above, one = 0;  // what lies above; a token's weight
      unsigned there = 0;         // tokens of the value
      for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) sh.radix_count[tid] = sh.radix_weight[0][tid] = sh.radix_weight[1][tid] = 0;
        __syncthreads();
        for (int v = r.v0 + lane; v < r.v1; v += 32) {
          const uint4 w = r.load(v);
          if (!(SmRow<X>::largest(SmRow<X>::more(SmRow<X>::start(), w)) >= reach)) continue;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const float x = SmRow<X>::at(w, e);
            const unsigned key = sm_key(x);
            if (!(x > -INFINITY) || !in_bin(x, v * E + e - r.skew) || (shift < 24 && (key ^ lo) >> (shift + 8) != 0)) continue;
            atomicAdd(&sh.radix_count[(key >> shift) & 255u], 1u);
            if (by_weight) sm_add(sh.radix_weight, (int)((key >> shift) & 255u), weight_of(x));
          }
        }
        sm_cluster_sync(cluster);
        if (tid < 256) {
          unsigned c = 0;
          u64 s = 0;
          for (int k = 0; k < cluster; ++k) c += sm_peer(&sh.radix_count[255 - tid], k), s += sm_peer(&sh.radix_weight[0][255 - tid], k) + ((u64)sm_peer(&sh.radix_weight[1][255 - tid], k) << 32);
          sh.merged_count[tid] = c;  // (from the largest digit down)
          sh.merged_weight[tid] = by_weight ? s : (u64)c;
        }
        if (tid == 0) sh.digit = -1;
        sm_cluster_sync(cluster);
        u64 sum;
        const u64 mine = tid < 256 ? sh.merged_weight[tid] : 0, first = sm_scan(mine, sh.scan, sum) + over;
        if (tid < 256 && sh.merged_count[tid] > 0 && (double)(first + mine) >= goal && (first == 0 || (double)first < goal)) {
          sh.digit = tid;
          sh.below = first;
        }
        __syncthreads();
        at = (unsigned)max(sh.digit, 0);  // (the step's sum reaches the goal, so a digit does)
        over = sh.below;
        there = sh.merged_count[at];
        one = there > 0 ? sh.merged_weight[at] / there : 0;
        lo |= (255u - at) << shift;
        __syncthreads();
      }
      // one value: all its tokens weigh the same, and as many of them as it takes are kept, the lowest indices
      unsigned ties = there;
      if (one > 0) {
        const double need = ceil((goal - (double)over) / (double)one);
        ties = need <= 1.0 ? 1u : need >= (double)there ? there : (unsigned)need;
      }
      unsigned mine = 0;
      const float lo_x = sm_value(lo);
      auto is_tie = [&](float x, int i) { return x == lo_x && in_bin(x, i); };
      for (int v = r.v0 + lane; v < r.v1; v += 32) {
        const uint4 w = r.load(v);
        if (!(SmRow<X>::largest(SmRow<X>::more(SmRow<X>::start(), w)) >= lo_x)) continue;
#pragma unroll
        for (int e = 0; e < E; ++e) mine += is_tie(SmRow<X>::at(w, e), v * E + e - r.skew) ? 1u : 0u;
      }
      mine = __reduce_add_sync(0xffffffffu, mine);
      if (lane == 0) sh.warp_ties[warp] = mine;
      if (tid == 0) sh.tie_index = -1;
      sm_cluster_sync(cluster);
      {
        unsigned seen = 0;  // ties before this warp's
        for (int i = lane; i < rank * kSmWarps + warp; i += 32) seen += sm_peer(&sh.warp_ties[i % kSmWarps], i / kSmWarps);
        seen = __reduce_add_sync(0xffffffffu, seen);
        if (seen < ties && seen + mine >= ties)
          for (int vb = r.v0; vb < r.v1; vb += 32) {  // the last kept one is among them
            const int v = vb + lane;
            unsigned hits = 0;
            if (v < r.v1) {
              const uint4 w = r.load(v);
#pragma unroll
              for (int e = 0; e < E; ++e) hits |= (is_tie(SmRow<X>::at(w, e), v * E + e - r.skew) ? 1u : 0u) << e;
            }
            const unsigned n = __popc(hits), upto = sm_warp_scan(n);
            unsigned place = seen + upto - n;
#pragma unroll
            for (int e = 0; e < E; ++e)
              if ((hits >> e) & 1u) {
                if (++place == ties) sh.tie_index = v * E + e - r.skew;
              }
            seen += __shfl_sync(0xffffffffu, upto, 31);
            if (seen >= ties) break;
          }
      }
      sm_cluster_sync(cluster);
      border.x = lo_x;
      border.index = -1;
      for (int k = 0; k < cluster; ++k) border.index = max(border.index, sm_peer(&sh.tie_index, k));
      sm_cluster_sync(cluster);
    }
    // ---- the kept weights, warp by warp; the token lies where their running sum passes the target
    if (least_x > border.x) border = SmBorder{least_x, 0x7fffffff};
    const bool uncut = border.x == -INFINITY;
    auto kept_weight = [&](float x, int i) { return uncut || border.keeps(x, i) ? weight_of(x) : 0ull; };
    auto sum_of = [&](int v0, int v1) {
      u64 s = 0;
      if (uncut)
        each_vector(r, v0, v1, [&](int, const uint4& w) {
#pragma unroll
          for (int e = 0; e < E; ++e) s += weight_of(SmRow<X>::at(w, e));
        });
      else each_vector(r, v0, v1, [&](int v, const uint4& w) {
        if (!(SmRow<X>::largest(SmRow<X>::more(SmRow<X>::start(), w)) >= border.x)) return;
#pragma unroll
        for (int e = 0; e < E; ++e) s += kept_weight(SmRow<X>::at(w, e), v * E + e - r.skew);
      });
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
      return s;
    };
    const u64 mine = sum_of(r.v0, r.v1);
    if (lane == 0) sh.warp_sum[warp] = mine;
    sm_cluster_sync(cluster);
    u64 all = 0, start = 0;
    int owner = 0;
    u64 target;
    {
      u64 s[kSmMaxCluster * kSmWarps / 32], sum = 0;  // neighbouring warps' sums per lane
      constexpr int N = kSmMaxCluster * kSmWarps / 32;
#pragma unroll
      for (int q = 0; q < N; ++q) {
        const int i = lane * N + q;
        s[q] = i < lists ? sm_peer(&sh.warp_sum[i % kSmWarps], i / kSmWarps) : 0ull;
        sum += s[q];
      }
      const u64 upto = sm_warp_scan(sum);
      all = __shfl_sync(0xffffffffu, upto, 31);
      target = min((u64)__double2ull_rd((double)u * (double)all), all - 1);
      u64 run = upto - sum;
      int found = -1;
#pragma unroll
      for (int q = 0; q < N; ++q) {
        if (found < 0 && run + s[q] > target) found = lane * N + q;
        if (found < 0) run += s[q];
      }
      const int who = __ffs(__ballot_sync(0xffffffffu, found >= 0)) - 1;
      owner = __shfl_sync(0xffffffffu, found, who);
      start = __shfl_sync(0xffffffffu, run, who);
    }
    if (owner / kSmWarps == rank) {
      // the owner's vectors in sixteenths, a warp each
      if (tid == (owner % kSmWarps) * 32) sh.offset[0] = (unsigned)r.v0, sh.offset[1] = (unsigned)r.v1;
      __syncthreads();
      const int o0 = (int)sh.offset[0], o1 = (int)sh.offset[1], per = (o1 - o0 + kSmWarps - 1) / kSmWarps;
      const int s0 = min(o1, o0 + warp * per), s1 = min(o1, s0 + per);
      const u64 part = sum_of(s0, s1);
      if (lane == 0) sh.scan[warp] = part;
      __syncthreads();
      u64 run = start;
      for (int w = 0; w < warp; ++w) run += sh.scan[w];
      if (run <= target && run + part > target)
        for (int vb = s0; vb < s1; vb += 32) {
          const int v = vb + lane;
          uint4 w = make_uint4(0u, 0u, 0u, 0u);
          u64 y[E], s = 0;
          if (v < s1) w = r.load(v);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            y[e] = v < s1 ? kept_weight(SmRow<X>::at(w, e), v * E + e - r.skew) : 0ull;
            s += y[e];
          }
          const u64 upto = sm_warp_scan(s);
          u64 at = run + upto - s;
          const bool here = at <= target && run + upto > target;
          if (here) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const bool was = at > target;
              at += y[e];
              if (!was && at > target) answer(v * E + e - r.skew, SmRow<X>::at(w, e), all);
            }
          }
          if (__any_sync(0xffffffffu, here)) break;
          run += __shfl_sync(0xffffffffu, upto, 31);
        }
    }
  }
  sm_cluster_sync(cluster);  // (no CTA ends while another reads from it)
}

constexpr size_t kSmSmemBytes = sizeof(SmShared);

}  // namespace dynts
