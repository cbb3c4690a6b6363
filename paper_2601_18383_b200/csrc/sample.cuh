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
// A cluster of CTAs takes a row, every warp a run of it.  What a row needs depends on its settings:
//   * top_k or top_p: few tokens decide.  Every lane keeps the maximum of what it read.  The r-th largest of a warp's 32 maxima
//     has r tokens of the warp at or above it, so with c the smallest of those values over the warps, 16 r tokens or more of the CTA
//     lie at or above c: with 16 r >= top_k the CTA's share of the top_k is among them.  The tokens from c on are collected
//     in a second reading (from L1 and L2), a list per warp and so in order; the first CTA merges the lists and decides alone.
//     For top_p the second reading also adds up all weights, and 16 r = 128 is tried; if the run is longer, or a list
//     overflows, or top_k is beyond 512, the row is
//   * selected by the whole cluster: three or four rounds of a histogram of 256 bins (tokens and weights) narrow the border down
//     to one value; a border inside equal values is a count of them.
//   * nothing cut off, or by min_p alone: no selection.
// Where the kept tokens are not in a list, the warps' sums of kept weights are exchanged and the one warp in whose run the
// token lies looks for it.
//
// Bound by the bytes of the logits for many rows (and by the exponentials where all weights are added up), by the
// chain load - maxima - second reading - exchange - decision for few.
#pragma once

#include "common.cuh"
#include "evict.cuh"  // the cluster barrier

namespace dynts {

constexpr int kSmThreads = 512;
constexpr int kSmWarps = kSmThreads / 32;
constexpr int kSmWarpList = 128;     // tokens a warp can collect
constexpr int kSmList = 4096;        // tokens the first CTA can merge
constexpr int kSmMaxCluster = 8;
constexpr int kSmTryP = 8;           // lanes' maxima per warp above the cut that top_p is tried with
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

struct SmHist {
  unsigned count[256];
  u64 weight[256];
};

// The border of a selection: values with a key above `key` are kept, and `ties` of those with it (the lowest indices).
struct SmCut {
  unsigned key, ties;
  u64 above, total;  // weights of the keys above it; with the ties
};

struct SmShared {
  double table[16];       // 2^(j / 16)
  float lane_cut[kSmWarps], warp_max[kSmWarps];
  unsigned warp_count[kSmWarps];
  u64 warp_sum[kSmWarps];
  unsigned warp_ties[kSmWarps];
  unsigned scan_u[kSmWarps];
  u64 scan_w[kSmWarps];
  // what the other CTAs of the cluster read
  float max, cut;
  u64 sum;                // of all weights, relative to this CTA's maximum
  int overflow;
  int verdict;            // of the first CTA: 1 the row is done
  unsigned peer_kmin;
  // selection
  int bin;
  u64 above;
  unsigned above_count;
  SmHist hist, merged;
  uint2 list[kSmWarps][kSmWarpList];  // key, index
};
struct SmMerged {  // of the first CTA of a cluster
  unsigned key[kSmList], index[kSmList];
  u64 weight[kSmList];
};

__device__ __forceinline__ void sm_cluster_sync() {  // (also of shared memory within the CTA)
  __syncwarp();
  cluster_arrive();
  cluster_wait();
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

__device__ __forceinline__ unsigned sm_key(float x) {  // order-preserving; -0 and +0 alike
  const unsigned b = __float_as_uint(x + 0.f);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float sm_value(unsigned key) { return __uint_as_float(key ^ ((key >> 31) ? 0x80000000u : 0xffffffffu)); }

// exp(y) for y <= 0 in units of 2^-45: e^y = 2^(n / 16) e^f with n whole and |f| <= ln 2 / 32; the series of e^f to f^6 is off by
// less than 5e-16 of it.  (y below -32, or not a number: less than half a unit, 0.)
__device__ __forceinline__ u64 sm_weight(double y, const double* table) {
  if (!(y > -32.0)) return 0;
  const double magic = 6755399441055744.0;  // 1.5 * 2^52: the sum's low bits are the whole part
  const double t = fma(y, 23.083120654223414, magic);  // 16 / ln 2
  const int n = __double2loint(t);
  const double f = fma(t - magic, -0.04332169878499658, y);  // ln 2 / 16
  double e = 1.0 / 720.0;
  e = fma(e, f, 1.0 / 120.0);
  e = fma(e, f, 1.0 / 24.0);
  e = fma(e, f, 1.0 / 6.0);
  e = fma(e, f, 0.5);
  e = fma(e, f, 1.0);
  e = fma(e, f, 1.0);
  e *= table[n & 15];
  e = __hiloint2double(__double2hiint(e) + (n >> 4) * (1 << 20), __double2loint(e));
  return (u64)__double_as_longlong(e + 128.0) - (u64)__double_as_longlong(128.0);  // (a unit of the sum's mantissa is 2^-45)
}

template <typename X>
struct SmRow {
  static constexpr int E = 16 / (int)sizeof(X);  // elements of a 16-byte vector
  const X* base;   // aligned down to 16 bytes
  int skew;        // elements between there and the row
  int vocab;
  int v0, v1;      // this warp's vectors
  // Vector v as floats; what lies outside the row is -inf, which weighs nothing.
  __device__ __forceinline__ void load(int v, float (&x)[E]) const {
    const int i = v * E - skew;
    if (i >= 0 && i + E <= vocab) {
      const uint4 w = *reinterpret_cast<const uint4*>(base + (size_t)v * E);
      if constexpr (E == 4) {
        x[0] = __uint_as_float(w.x), x[1] = __uint_as_float(w.y), x[2] = __uint_as_float(w.z), x[3] = __uint_as_float(w.w);
      } else {
        const unsigned y[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[2 * e] = __uint_as_float(y[e] << 16), x[2 * e + 1] = __uint_as_float(y[e] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = i + e >= 0 && i + e < vocab ? to_float(base[(size_t)v * E + e]) : -INFINITY;
    }
  }
};

__device__ __forceinline__ float sm_max_nan(float a, float b) {  // a NaN stays
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

// The border by count (pz < 0: the first `want` are kept) or by weight (the shortest run that reaches pz).  each(f) calls
// f(key, weight()) for the tokens of this CTA; with `cluster` > 1 the histograms of all its CTAs are added up.
template <typename Each>
__device__ SmCut sm_select(SmShared& sh, Each each, int cluster, unsigned kmin, unsigned kmax, unsigned want, double pz) {
  const int tid = threadIdx.x, lane = tid & 31;
  const bool by_weight = pz >= 0.0;
  int shift = max(0, 24 - __clz(kmax - kmin));
  unsigned lo = kmin, bins = 256, above_count = 0, here = 0;
  u64 above = 0, here_w = 0;
  while (true) {
    for (int i = tid; i < 256; i += kSmThreads) sh.hist.count[i] = 0, sh.hist.weight[i] = 0;
    __syncthreads();
    each([&](unsigned key, auto weight) {
      const unsigned at = (key - lo) >> shift;
      if (key < lo || at >= bins) return;
      atomicAdd(&sh.hist.count[at], 1u);
      const u64 w = weight();
      if (w) atomicAdd(&sh.hist.weight[at], w);
    });
    if (cluster > 1) {
      sm_cluster_sync();
      if (tid < 256) {
        unsigned c = 0;
        u64 w = 0;
        for (int r = 0; r < cluster; ++r) c += sm_peer(&sh.hist.count[tid], r), w += sm_peer(&sh.hist.weight[tid], r);
        sh.merged.count[tid] = c;
        sh.merged.weight[tid] = w;
      }
      sm_cluster_sync();  // (the histograms have been read)
    } else {
      __syncthreads();
    }
    const SmHist& h = cluster > 1 ? sh.merged : sh.hist;
    if (tid < 32) {  // from the top bin down, eight per lane
      unsigned c = 0;
      u64 w = 0;
      const int top = 255 - 8 * lane;
      for (int k = 0; k < 8; ++k) c += h.count[top - k], w += h.weight[top - k];
      unsigned cs = c;
      u64 ws = w;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned c2 = __shfl_up_sync(0xffffffffu, cs, o);
        const u64 w2 = __shfl_up_sync(0xffffffffu, ws, o);
        if (lane >= o) cs += c2, ws += w2;
      }
      u64 aw = above + ws - w;
      unsigned ac = above_count + cs - c;
      int bin = -1;
      for (int k = 0; k < 8 && bin < 0; ++k) {
        const unsigned hc = h.count[top - k];
        const u64 hw = h.weight[top - k];
        if (hc > 0 && (by_weight ? (double)(aw + hw) >= pz : ac + hc >= want)) bin = top - k;
        else ac += hc, aw += hw;
      }
      const unsigned found = __ballot_sync(0xffffffffu, bin >= 0);
      // (the sums reach their own total; were it missed by a rounding, everything is kept)
      if (found == 0 ? lane == 31 : lane == __ffs(found) - 1) {
        sh.bin = bin;
        sh.above = aw;
        sh.above_count = ac;
      }
    }
    __syncthreads();
    const int bin = sh.bin;
    above = sh.above;
    above_count = sh.above_count;
    if (bin < 0) {
      __syncthreads();
      return SmCut{0u, 0u, above, above};  // every key is above 0
    }
    here = h.count[bin];
    here_w = h.weight[bin];
    lo += (unsigned)bin << shift;
    __syncthreads();
    if (shift == 0) break;
    const int next = max(0, shift - 8);
    bins = 1u << (shift - next);
    shift = next;
  }
  // one value: all its tokens weigh the same
  const u64 w = here_w / here;
  unsigned ties = want - above_count;
  if (by_weight) {
    ties = here;
    if (w > 0) {
      const double need = (pz - (double)above) / (double)w;
      ties = need <= 1.0 ? 1u : need >= (double)here ? here : (unsigned)ceil(need);
    }
  }
  return SmCut{lo, ties, above, above + w * ties};
}

// The running sum of a value over the CTA's threads (exclusive); every thread gets the total.
template <typename V>
__device__ __forceinline__ V sm_scan(V x, V* warps, V& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  V s = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const V y = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += y;
  }
  __syncthreads();
  if (lane == 31) warps[warp] = s;
  __syncthreads();
  V before = 0;
  total = 0;
  for (int w = 0; w < kSmWarps; ++w) {
    if (w < warp) before += warps[w];
    total += warps[w];
  }
  return before + s - x;
}

template <typename X>
__global__ void __launch_bounds__(kSmThreads) sample_kernel(const __grid_constant__ SampleParams p) {
  constexpr int E = SmRow<X>::E;
  extern __shared__ __align__(16) uint8_t sm_raw[];
  SmShared& sh = *reinterpret_cast<SmShared*>(sm_raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int cluster = p.cluster, row = (int)blockIdx.x / cluster, rank = (int)blockIdx.x - row * cluster;

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
  const double inv_t = 1.0 / (double)T;
  const int tries = top_k > 0 ? (top_k + kSmWarps - 1) / kSmWarps : kSmTryP;  // lanes' maxima per warp
  const bool listed = (top_k > 0 || cut_p) && tries <= 32;
  if (tid < 16) sh.table[tid] = exp2((double)tid / 16.0);
  if (tid == 0) sh.overflow = listed ? 0 : 1, sh.verdict = 0;

  // ---- every lane's maximum
  float top = -INFINITY;
#pragma unroll 4
  for (int v = r.v0 + lane; v < r.v1; v += 32) {
    float x[E];
    r.load(v, x);
#pragma unroll
    for (int e = 0; e < E; ++e) top = sm_max_nan(top, x[e]);
  }
  {
    float s = top;  // sorted over the lanes, the largest first (a NaN makes the row's answer void below)
    if (listed) {
#pragma unroll
      for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
        for (int o = k >> 1; o > 0; o >>= 1) {
          const float y = __shfl_xor_sync(0xffffffffu, s, o);
          s = ((lane & k) == 0) == ((lane & o) == 0) ? fmaxf(s, y) : fminf(s, y);
        }
    }
    const float cut = __shfl_sync(0xffffffffu, s, min(tries, 32) - 1);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = sm_max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
    if (lane == 0) sh.lane_cut[warp] = cut, sh.warp_max[warp] = top;
  }
  __syncthreads();
  float cut = sh.lane_cut[0];
  top = sh.warp_max[0];
#pragma unroll
  for (int w = 1; w < kSmWarps; ++w) cut = fminf(cut, sh.lane_cut[w]), top = sm_max_nan(top, sh.warp_max[w]);
  if (tid == 0) sh.max = top, sh.cut = cut;

  // ---- the tokens from the cut on, and all weights where top_p needs their sum (relative to this CTA's maximum)
  if (listed) {
    const bool sum_all = cut_p && top_k == 0;
    unsigned count = 0;
    u64 sum = 0;
    const double top_d = (double)top;
    for (int vb = r.v0; vb < r.v1; vb += 32) {
      const int v = vb + lane;
      float x[E];
      float best = -INFINITY;
      if (v < r.v1) {
        r.load(v, x);
#pragma unroll
        for (int e = 0; e < E; ++e) best = fmaxf(best, x[e]);
        if (sum_all) {
#pragma unroll
          for (int e = 0; e < E; ++e) sum += sm_weight(((double)x[e] - top_d) * inv_t, sh.table);
        }
      }
      const bool any = v < r.v1 && best >= cut && best > -INFINITY;
      if (!__any_sync(0xffffffffu, any)) continue;
      unsigned hits = 0;  // a bit for each of the lane's elements
      if (any) {
#pragma unroll
        for (int e = 0; e < E; ++e) hits |= (x[e] >= cut && x[e] > -INFINITY ? 1u : 0u) << e;
      }
      const unsigned n = __popc(hits);
      unsigned at = n;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned y = __shfl_up_sync(0xffffffffu, at, o);
        if (lane >= o) at += y;
      }
      const unsigned all = __shfl_sync(0xffffffffu, at, 31);
      at += count - n;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if ((hits >> e) & 1u) {
          if (at < kSmWarpList) sh.list[warp][at] = make_uint2(sm_key(x[e]), (unsigned)(v * E + e - r.skew));
          ++at;
        }
      count += all;
    }
    if (count > kSmWarpList) sh.overflow = 1;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sh.warp_count[warp] = min(count, (unsigned)kSmWarpList), sh.warp_sum[warp] = sum;
    __syncthreads();
    if (tid == 0) {
      u64 s = 0;
      for (int w = 0; w < kSmWarps; ++w) s += sh.warp_sum[w];
      sh.sum = s;
    }
  }
  if (cluster > 1) {
    sm_cluster_sync();
  } else {
    __syncthreads();
  }
  float M = -INFINITY;
  float cut_all = -INFINITY;
  bool overflow = false;
  for (int k = 0; k < cluster; ++k) {
    M = sm_max_nan(M, sm_peer(&sh.max, k));
    cut_all = fmaxf(cut_all, sm_peer(&sh.cut, k));
    overflow = overflow || sm_peer(&sh.overflow, k) != 0;
  }
  const double Md = (double)M;
  const bool no_answer = !(M > -INFINITY && M < INFINITY);  // NaN or +inf somewhere, or nothing but -inf
  const double x_min = min_p > 0.f ? Md + (double)T * log((double)min_p) : -INFINITY;  // (min_p > 1: nothing but the maximum is kept)
  auto weight_of = [&](float x) { return sm_weight(((double)x - Md) * inv_t, sh.table); };
  auto answer = [&](int token, float x, u64 total) {
    p.tokens[row] = token;
    if (p.logprobs) p.logprobs[row] = (float)(((double)x - Md) * inv_t - log((double)total * 2.842170943040401e-14));  // 2^-45
  };
  if (no_answer) {
    if (rank == 0 && tid == 0) {
      p.tokens[row] = -1;
      if (p.logprobs) p.logprobs[row] = NAN;
    }
  } else {
    const double low = fmin(x_min, Md);
    bool done = false;
    if (!overflow) {
      // ---- the first CTA merges the lists and decides
      if (rank == 0) {
        SmMerged& m = *reinterpret_cast<SmMerged*>(sm_raw + ((sizeof(SmShared) + 15) & ~(size_t)15));
        unsigned base = 0;
        unsigned kmax = sm_key(M);
        double total = 0.0;
        for (int k = 0; k < cluster; ++k) {
          unsigned before = base;
          for (int w = 0; w < kSmWarps; ++w) {
            const unsigned c = sm_peer(&sh.warp_count[w], k);
            if (w < warp) before += c;
            base += c;
          }
          const unsigned c = sm_peer(&sh.warp_count[warp], k);
          for (unsigned i = lane; i < c; i += 32) {
            const uint2 y = sm_peer(&sh.list[warp][i], k);
            if (before + i < kSmList) {
              m.key[before + i] = y.x;
              m.index[before + i] = y.y;
              m.weight[before + i] = weight_of(sm_value(y.x));
            }
          }
          if (cut_p && top_k == 0) total += (double)sm_peer(&sh.sum, k) * exp(((double)sm_peer(&sh.max, k) - Md) * inv_t);
        }
        const unsigned n = base, kcut = sm_key(cut_all);
        __syncthreads();
        bool fits = n <= kSmList;
        if (fits) {
          auto each = [&](auto f) {
            for (unsigned i = tid; i < n; i += kSmThreads) {
              const unsigned key = m.key[i];
              f(key, [&]() { return m.weight[i]; });
            }
          };
          SmCut c{0u, 0u, 0, 0};
          if (top_k > 0) {
            c = sm_select(sh, each, 1, kcut, kmax, (unsigned)top_k, -1.0);
            total = (double)c.total;
          }
          if (cut_p) {
            // (of the tokens below the cut some are missing; of those from top_k on nothing counts)
            const SmCut q = sm_select(sh, each, 1, top_k > 0 ? max(c.key, kcut) : kcut, kmax, 0u, (double)top_p * total);
            if (q.key == 0u) {
              if (top_k == 0) fits = false;  // the run is longer than the list
            } else {
              const unsigned ties = top_k > 0 && q.key == c.key ? min(q.ties, c.ties) : q.ties;
              c = q;
              c.ties = ties;
            }
          }
          if (fits) {
            // the kept tokens' running sums, in the order of the vocabulary: a run of the list per thread
            const unsigned per = (n + kSmThreads - 1) / kSmThreads, i0 = min(n, tid * per), i1 = min(n, i0 + per);
            unsigned ties = 0, all_ties;
            for (unsigned i = i0; i < i1; ++i) ties += m.key[i] == c.key;
            const unsigned ties0 = sm_scan(ties, sh.scan_u, all_ties);
            auto kept = [&](unsigned i, unsigned& seen) {
              const unsigned key = m.key[i];
              const bool tie = key == c.key;
              const bool yes = (key > c.key || (tie && seen < c.ties)) && (double)sm_value(key) >= low;
              seen += tie;
              return yes ? m.weight[i] : 0ull;
            };
            u64 mine = 0, all;
            unsigned seen = ties0;
            for (unsigned i = i0; i < i1; ++i) mine += kept(i, seen);
            u64 run = sm_scan(mine, sh.scan_w, all);
            const u64 target = min((u64)__double2ull_rd((double)u * (double)all), all - 1);
            if (run <= target && run + mine > target) {
              seen = ties0;
              for (unsigned i = i0; i < i1; ++i) {
                run += kept(i, seen);
                if (run > target) {
                  answer((int)m.index[i], sm_value(m.key[i]), all);
                  break;
                }
              }
            }
          }
        }
        if (tid == 0) sh.verdict = fits ? 1 : 0;
        __syncthreads();
      }
      if (cluster > 1) {
        sm_cluster_sync();
        done = sm_peer(&sh.verdict, 0) != 0;
      } else {
        done = sh.verdict != 0;
      }
    }
    if (!done) {
      // ---- the whole row
      SmCut c{0u, 0u, 0, 0};
      auto each = [&](auto f) {
        for (int v = r.v0 + lane; v < r.v1; v += 32) {
          float x[E];
          r.load(v, x);
#pragma unroll
          for (int e = 0; e < E; ++e)
            if (x[e] > -INFINITY) f(sm_key(x[e]), [&]() { return weight_of(x[e]); });
        }
      };
      const unsigned kmax = sm_key(M), kmin = 0x00800000u;  // (finite values)
      auto kept_sums = [&](u64& sum, unsigned& ties) {  // of this warp: weights above the border, tokens on it
        sum = 0;
        ties = 0;
        for (int v = r.v0 + lane; v < r.v1; v += 32) {
          float x[E];
          r.load(v, x);
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const unsigned key = sm_key(x[e]);
            if (key > c.key && (double)x[e] >= low) sum += weight_of(x[e]);
            ties += key == c.key ? 1u : 0u;
          }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o), ties += __shfl_xor_sync(0xffffffffu, ties, o);
      };
      auto exchange = [&]() {
        if (cluster > 1) {
          sm_cluster_sync();
        } else {
          __syncthreads();
        }
      };
      double total = 0.0;
      if (top_k > 0) {
        c = sm_select(sh, each, cluster, kmin, kmax, (unsigned)top_k, -1.0);
        if (c.key == 0u) c = SmCut{0u, 0u, 0, 0};  // (fewer finite tokens than top_k)
        total = (double)c.total;
      }
      if (cut_p) {
        if (top_k == 0) {
          u64 s = 0;
          each([&](unsigned, auto weight) { s += weight(); });
#pragma unroll
          for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
          if (lane == 0) sh.warp_sum[warp] = s;
          exchange();
          u64 z = 0;
          for (int k = 0; k < cluster; ++k)
            for (int w = 0; w < kSmWarps; ++w) z += sm_peer(&sh.warp_sum[w], k);
          total = (double)z;
          exchange();
        }
        const SmCut q = sm_select(sh, each, cluster, max(kmin, c.key), kmax, 0u, (double)top_p * total);
        if (q.key != 0u) {
          const unsigned ties = top_k > 0 && q.key == c.key ? min(q.ties, c.ties) : q.ties;
          c = q;
          c.ties = ties;
        }
      }
      u64 sum;
      unsigned ties;
      kept_sums(sum, ties);
      if (lane == 0) sh.warp_sum[warp] = sum, sh.warp_ties[warp] = ties;
      exchange();
      // the warps' sums in order; a tie counts while fewer than c.ties lie before it
      const float tie_x = sm_value(c.key);
      const u64 tie_w = c.ties > 0 && (double)tie_x >= low ? weight_of(tie_x) : 0;
      u64 all = 0, before = 0;
      unsigned seen = 0, seen_mine = 0;
      for (int k = 0; k < cluster; ++k)
        for (int w = 0; w < kSmWarps; ++w) {
          if (k == rank && w == warp) before = all, seen_mine = seen;
          const unsigned t = sm_peer(&sh.warp_ties[w], k), take = seen < c.ties ? min(t, c.ties - seen) : 0u;
          all += sm_peer(&sh.warp_sum[w], k) + tie_w * take;
          seen += t;
        }
      const u64 mine = sum + tie_w * (seen_mine < c.ties ? min(ties, c.ties - seen_mine) : 0u);
      const u64 target = min((u64)__double2ull_rd((double)u * (double)all), all - 1);
      if (before <= target && before + mine > target) {
        // the token lies in this warp's run
        u64 run = before;
        bool found = false;
        for (int vb = r.v0; vb < r.v1 && !found; vb += 32) {
          const int v = vb + lane;
          float x[E];
          unsigned keys[E], t = 0;
          if (v < r.v1) {
            r.load(v, x);
          } else {
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = -INFINITY;
          }
#pragma unroll
          for (int e = 0; e < E; ++e) keys[e] = sm_key(x[e]), t += keys[e] == c.key ? 1u : 0u;
          unsigned ts = t;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const unsigned y = __shfl_up_sync(0xffffffffu, ts, o);
            if (lane >= o) ts += y;
          }
          unsigned at = seen_mine + ts - t;
          u64 w[E], s = 0;
#pragma unroll
          for (int e = 0; e < E; ++e) {
            const bool tie = keys[e] == c.key;
            w[e] = keys[e] > c.key && (double)x[e] >= low ? weight_of(x[e]) : tie && at < c.ties ? tie_w : 0ull;
            at += tie ? 1u : 0u;
            s += w[e];
          }
          u64 ss = s;
#pragma unroll
          for (int o = 1; o < 32; o <<= 1) {
            const u64 y = __shfl_up_sync(0xffffffffu, ss, o);
            if (lane >= o) ss += y;
          }
          u64 mine_run = run + ss - s;
          const bool here = mine_run <= target && run + ss > target;
          if (here) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const bool was = mine_run > target;
              mine_run += w[e];
              if (!was && mine_run > target) answer(v * E + e - r.skew, x[e], all);
            }
          }
          found = __any_sync(0xffffffffu, here);
          run += __shfl_sync(0xffffffffu, ss, 31);
          seen_mine += __shfl_sync(0xffffffffu, ts, 31);
        }
      }
    }
  }
  if (cluster > 1) {
    sm_cluster_sync();  // (no CTA ends while another reads from it)
  }
}

constexpr size_t kSmSmemBytes = ((sizeof(SmShared) + 15) & ~(size_t)15) + sizeof(SmMerged);

}  // namespace dynts
