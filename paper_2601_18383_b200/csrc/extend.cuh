// A chunk of new tokens per sequence against the rows a cache holds (Eq. 4-6 for several queries at
// once): the rows are stored behind the sequence's end, token i of a chunk that begins at row n
// attends to the rows [0, n + i], and -- if wanted -- every row receives the attention mass the
// chunk's queries gave it.  This file holds what every shape shares (parameters, the definition of
// a logit and of visibility, the kernel that stores the rows and publishes the lengths) and the
// fp32-FMA kernels that serve every type and head size; extend_tc.cuh holds the tensor-core kernels
// for head_dim 128.
//
// Definitions, for query token i of a sequence and row j (p = positions, kept by rows that survive
// an eviction):
//   x   = q_i . k_j / sqrt(d)
//   x   = c tanh(x / c)                      if a cap c > 0 is given
//   x  -= slope_h |p_i - p_j|                if slopes are given
//   row j is visible  <=>  j <= n + i, or j is one of the chunk's first `prefix` rows;
//                          and |p_i - p_j| < window, if a window is given
// A token always sees itself, so no row of weights is empty.  (A logit of -inf weighs nothing; a token whose visible
// logits are all -inf has no answer: NaN.)  All logits are kept in base-2 units
// (times log2 e), sums and maxima in fp32.
#pragma once

#include <math_constants.h>

#include "common.cuh"
#include "evict.cuh"  // the cluster barrier

namespace dynts {

constexpr int kExtSeqs = 128;          // sequences of one launch (a larger batch takes several)
constexpr int kExtGenericRows = 32;    // query rows (token, head of the group) per CTA of the generic kernel
constexpr int kExtGenericKeys = 32;    // keys per tile of the generic kernels
constexpr int kExtGenericThreads = 256;
constexpr int kExtTileKeys = 64;       // keys per tile of the tensor-core kernel; rows up to its end are zeroed behind the chunk

struct ExtendSeqs {
  int n;                          // sequences of this launch, b0 .. b0 + n - 1
  int b0;
  int tok0[kExtSeqs + 1];         // first packed token of each (the chunk of sequence s: tok0[s] .. tok0[s + 1] - 1)
  int item0[kExtSeqs + 1];        // first work item of each (what an item is depends on the kernel)
  int prefix[kExtSeqs];           // leading tokens of the chunk that every token of the chunk sees
};

struct ExtendParams {
  const void* q;      // [n_layers][total][Hq][d], token stride q_stride elements
  const void* k;      // [n_layers][total][Hkv][d]
  const void* v;
  void* out;          // [n_layers][total][Hq][d], contiguous
  long long q_stride, k_stride, v_stride;
  void* K;            // full [L, Nb, Hkv, cap, d]
  void* V;
  int* pos;
  float* score;
  float* comp;
  int* len;           // [Nb]
  int* tot;
  int* active;
  int* err;
  unsigned int* ticket;
  const float* s_new; // [total] scores of the new rows, or NULL: 0
  float* lse;         // [n_layers][Hkv][total][G] log2 of the sum of the weights' exponentials, or NULL
  float* mass;        // full [L, Nb, Hkv, cap], or NULL
  const float* slopes;  // [Hq] or NULL
  int layer0, n_layers, total;
  int Nb, Hq, Hkv, G, d, cap;
  int window;         // 0: none
  int publish;        // the storing kernel advances the lengths when it is done
  int* held;          // [2][kExtSeqs], written by the storing kernel: rows held before the chunk (-1: it does not fit), tokens seen before it
  int accumulate;     // the mass is added to the scores
  __half* q16;        // 8-bit rows: [n_layers][total][Hq][d] f16 copies of the queries made by the storing kernel, or NULL
  unsigned int* counters;  // words the storing kernel clears for the kernel behind it
  int n_counters;
  int zero_tail;      // the storing kernel clears the V rows from the chunk's end to the end of the key tile
  float scale;        // 1 / sqrt(d), times k_scale for 8-bit rows
  float cap_logit;    // c, or 0
  float k_scale, v_scale;  // 8-bit rows
  ExtendSeqs seqs;
};

// The tensor-core kernel's work, laid out by the storing kernel (which knows the lengths on the device and runs before
// it anyway): an item = (tile of query rows, KV head, layer, sequence); all items' key tiles form one list, of which
// every CTA takes an equal contiguous piece.  The list is kept in shares: an item of sequence s counts per[s] shares
// whatever its exact number of key tiles, a share's border inside an item is the same fraction of its key tiles.
// CTA c takes the shares [c * q + min(c, rem), ...).  What CTA c does of item i is described by 32 words at slot i + c
// (an item's parts and a CTA's pieces both lie side by side).
constexpr int kPlanWords = 32;
enum PlanWord { kPwTiles, kPwFirst, kPwTok, kPwLayer, kPwHead, kPwHeld, kPwTok0, kPwRows, kPwNew, kPwSlab, kPwParts, kPwPlace, kPwBase, kPwList, kPwPrefix, kPwSeen };
struct ExtendPlan {
  unsigned cum[kExtSeqs + 1];  // shares before each sequence's first item
  unsigned per[kExtSeqs];      // shares of an item
  int tiles[kExtSeqs];         // tiles of query rows per (layer, KV head)
  int item0[kExtSeqs + 1];     // items before each sequence's
  unsigned share_q, share_rem; // shares per CTA: share_q, one more for the first share_rem
  int tokens_per_tile;         // floor(128 / G)
  int lh;                      // n_layers * Hkv
  int* words;                  // [items + CTAs][kPlanWords], or NULL: no plan is wanted
};
__device__ __forceinline__ unsigned plan_share0(const ExtendPlan& p, unsigned cta) { return cta * p.share_q + min(cta, p.share_rem); }
__device__ __forceinline__ unsigned plan_cta_of(const ExtendPlan& p, unsigned share) {
  const unsigned big = p.share_rem * (p.share_q + 1u);
  return share < big ? share / (p.share_q + 1u) : p.share_rem + (share - big) / p.share_q;
}
__device__ __forceinline__ int plan_item_of(const ExtendPlan& p, int n_seq, unsigned share) {
  int lo = 0, hi = n_seq;
  while (hi - lo > 1) {  // the last sequence that begins at or before the share
    const int mid = (lo + hi) >> 1;
    if (p.cum[mid] <= share) lo = mid;
    else hi = mid;
  }
  return p.item0[lo] + (int)((share - p.cum[lo]) / p.per[lo]);
}
// total * a / per, in 32 bits where that is enough (a 64-bit division takes several hundred cycles)
__device__ __forceinline__ int plan_part(unsigned total, unsigned a, unsigned per) {
  return (int)((total | a) < 65536u ? total * a / per : (unsigned)((unsigned long long)total * a / per));
}

__device__ __forceinline__ int ext_find(const int* first, int n, int x) {  // the s with first[s] <= x < first[s + 1]
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Where the log-sum-exps of a packed token's query rows begin: a KV head's rows (token, head of the group) adjoin.
__device__ __forceinline__ size_t ext_lse_index(const ExtendParams& p, int layer, int h, int tok) {
  return (((size_t)layer * p.Hkv + h) * p.total + tok) * p.G;
}

// Rows held and tokens seen before the chunk, as the storing kernel found them: the lengths may include the chunk by now,
// and a sequence whose chunk did not fit (a replayed graph's may have grown) has kept its length.
struct ExtSeq {
  int b, t, n, tot;
  bool ok;  // the chunk fits the slab
};
__device__ __forceinline__ ExtSeq ext_seq(const ExtendParams& p, int s) {
  ExtSeq e;
  e.b = p.seqs.b0 + s;
  e.t = p.seqs.tok0[s + 1] - p.seqs.tok0[s];
  e.n = p.held[s];
  e.tot = p.held[kExtSeqs + s];
  e.ok = e.n >= 0;
  return e;
}

// The tensor-core kernel's plan: a warp per item, a lane per part.
__device__ __forceinline__ void ext_write_plan(const ExtendParams& p, const ExtendPlan& q, int warp, int n_warps) {
  const int lane = threadIdx.x & 31;
  for (int item = warp; item < q.item0[p.seqs.n]; item += n_warps) {
    const int s = ext_find(q.item0, p.seqs.n, item);
    const int idx = item - q.item0[s], nq = q.tiles[s], lh = idx / nq, o = idx - lh * nq;
    // tiles from both ends in turn: neighbours in the list hold about as many key tiles together as any other two
    const int qt = (o & 1) ? nq - 1 - (o >> 1) : o >> 1;
    const int b = p.seqs.b0 + s, t = p.seqs.tok0[s + 1] - p.seqs.tok0[s], n = p.len[b], prefix = p.seqs.prefix[s];
    const int i0 = qt * q.tokens_per_tile, i1 = min(t, i0 + q.tokens_per_tile);
    const bool ok = n >= 0 && n + t <= p.cap;  // (else nothing is stored and nothing computed)
    const int seen = n + max(i1, prefix);
    // (positions ascend with the rows, so a row more than `window` rows back is more than `window` positions back)
    const int first = p.window > 0 ? max(0, n + i0 - p.window + 1) / kExtTileKeys : 0;
    const int total = (seen + kExtTileKeys - 1) / kExtTileKeys - first;
    const unsigned per = q.per[s], start = q.cum[s] + (unsigned)idx * per;
    const unsigned ca = plan_cta_of(q, start), cb = plan_cta_of(q, start + per - 1u);
    const int layer = lh / p.Hkv, h = lh - layer * p.Hkv;
    int count = 0;
    for (int pass = 0; pass < 2; ++pass) {  // how many parts hold any key tile; then the words
      int rank = 0;
      for (unsigned c0 = ca; c0 <= cb; c0 += 32) {
        const unsigned c = c0 + (unsigned)lane;
        int lo = 0, hi = 0;
        if (c <= cb && ok) {
          const unsigned v0 = plan_share0(q, c), v1 = plan_share0(q, c + 1u);
          const unsigned a = v0 > start ? v0 - start : 0u, e = v1 - start < per ? v1 - start : per;
          lo = a == 0u ? 0 : plan_part((unsigned)total, a, per);
          hi = e == per ? total : plan_part((unsigned)total, e, per);
        }
        const unsigned has = __ballot_sync(0xffffffffu, lo < hi);
        if (pass == 1 && c <= cb) {
          int* w = q.words + (size_t)(item + (int)c) * kPlanWords;
          // A CTA has two places for parts: one for an item that began before its shares, one for an item that begins in them.
          const int place = (int)(2u * c) + (c == ca ? 1 : 0);
          if (lo < hi) q.words[(size_t)(item + (int)ca + rank + __popc(has & ((1u << lane) - 1u))) * kPlanWords + kPwList] = place;
          w[kPwTiles] = hi - lo;
          w[kPwFirst] = first + lo;
          w[kPwTok] = p.seqs.tok0[s] + i0;
          w[kPwLayer] = layer;
          w[kPwHead] = h;
          w[kPwHeld] = n;
          w[kPwTok0] = i0;
          w[kPwRows] = (i1 - i0) * p.G;
          w[kPwNew] = t;
          w[kPwSlab] = ((p.layer0 + layer) * p.Nb + b) * p.Hkv + h;
          w[kPwParts] = count;
          w[kPwPlace] = place;
          w[kPwBase] = item + (int)ca;
          w[kPwPrefix] = prefix;
          w[kPwSeen] = p.tot[b];
        }
        rank += __popc(has);
      }
      count = rank;
    }
  }
}

// Stores the chunk's rows: K and V (encoded for 8-bit slabs), position, score; with `publish` the
// last CTA to finish advances the lengths.  Short: a row is read and written once, and
// what it takes (3 to 5 us for up to a few thousand rows) is the latency of a launch, of the lengths and of the plan's words.
// Grid: x over the 16-byte pieces of the tokens' rows, y over (layer, KV head).
template <typename T, bool KV8>
__global__ void __launch_bounds__(256) extend_store_kernel(const __grid_constant__ ExtendParams p, const __grid_constant__ ExtendPlan plan) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the next kernel's set-up may begin; it waits for this grid before it reads
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr int E = 16 / (int)sizeof(T);  // elements per 16-byte piece of the source
  const unsigned pieces = (unsigned)p.d / E;
  const int tok_begin = p.seqs.tok0[0];
  const unsigned n_tok = (unsigned)(p.seqs.tok0[p.seqs.n] - tok_begin);
  const unsigned stride = gridDim.x * blockDim.x, first = blockIdx.x * blockDim.x + threadIdx.x;
  const int layer = blockIdx.y / p.Hkv, h = blockIdx.y - layer * p.Hkv;
  const size_t slab0 = (size_t)(p.layer0 + layer) * p.Nb;  // (times Hkv, plus the sequence's and head's part)
  for (unsigned w = first; w < n_tok * pieces; w += stride) {
    const unsigned rel = w / pieces, piece = w - rel * pieces;
    const int tok = tok_begin + (int)rel;
    const int s = ext_find(p.seqs.tok0, p.seqs.n, tok);
    const int b = p.seqs.b0 + s, t = p.seqs.tok0[s + 1] - p.seqs.tok0[s], i = tok - p.seqs.tok0[s];
    const size_t src_tok = (size_t)layer * p.total + tok;
    const uint4 kk = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.k) + src_tok * p.k_stride + (size_t)h * p.d + piece * E);
    const uint4 vv = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.v) + src_tok * p.v_stride + (size_t)h * p.d + piece * E);
    const int n = p.len[b];
    if (n < 0 || n + t > p.cap) {
      if (piece == 0 && h == 0 && i == 0) atomicOr(p.err, kErrLenOverflow);
      continue;
    }
    const size_t row = ((slab0 + b) * p.Hkv + h) * p.cap + n + i;
    if constexpr (KV8) {
      const __nv_bfloat16* kx = reinterpret_cast<const __nv_bfloat16*>(&kk);
      const __nv_bfloat16* vx = reinterpret_cast<const __nv_bfloat16*>(&vv);
      uint32_t kc[2] = {0u, 0u}, vc[2] = {0u, 0u};
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        kc[u >> 2] |= (uint32_t)store_e4m3(__bfloat162float(kx[u]), p.k_scale) << (8 * (u & 3));
        vc[u >> 2] |= (uint32_t)store_e4m3(__bfloat162float(vx[u]), p.v_scale) << (8 * (u & 3));
      }
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.K) + row * p.d + piece * 8) = make_uint2(kc[0], kc[1]);
      *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.V) + row * p.d + piece * 8) = make_uint2(vc[0], vc[1]);
    } else {
      *reinterpret_cast<uint4*>(static_cast<T*>(p.K) + row * p.d + piece * E) = kk;
      *reinterpret_cast<uint4*>(static_cast<T*>(p.V) + row * p.d + piece * E) = vv;
    }
    if (piece == 0) {
      p.pos[row] = p.tot[b] + i;
      p.score[row] = p.s_new ? p.s_new[tok] : 0.f;
      p.comp[row] = 0.f;
    }
  }
  if (blockIdx.x == 0 && blockIdx.y == 0)
    for (int s = threadIdx.x; s < p.seqs.n; s += blockDim.x) {
      const int b = p.seqs.b0 + s, n = p.len[b];
      p.held[s] = n >= 0 && n + p.seqs.tok0[s + 1] - p.seqs.tok0[s] <= p.cap ? n : -1;
      p.held[kExtSeqs + s] = p.tot[b];
    }
  if (plan.words) {
    const int warps = (int)(gridDim.x * gridDim.y * blockDim.x / 32);
    ext_write_plan(p, plan, (int)((blockIdx.y * gridDim.x + blockIdx.x) * (blockDim.x / 32) + threadIdx.x / 32), warps);
  }
  if (blockIdx.y == 0)
    for (unsigned w = first; w < (unsigned)p.n_counters; w += stride) p.counters[w] = 0u;
  if constexpr (KV8) {
    if (p.q16) {  // (8-bit codes are exact in f16, and both operands of an MMA have one type)
      const unsigned qp = (unsigned)p.d / 8, per_tok = (unsigned)p.G * qp;
      for (unsigned w = first; w < n_tok * per_tok; w += stride) {
        const unsigned rel = w / per_tok, y = w - rel * per_tok;  // the group's heads adjoin
        const size_t tok = (size_t)layer * p.total + tok_begin + rel, col = (size_t)h * p.G * p.d + y * 8;
        const uint4 x = *reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + tok * p.q_stride + col);
        const __nv_bfloat162* b2 = reinterpret_cast<const __nv_bfloat162*>(&x);
        uint4 o;
        __half2* h2 = reinterpret_cast<__half2*>(&o);
#pragma unroll
        for (int u = 0; u < 4; ++u) h2[u] = __float22half2_rn(__bfloat1622float2(b2[u]));
        *reinterpret_cast<uint4*>(p.q16 + tok * p.Hq * p.d + col) = o;
      }
    }
  }
  if (p.zero_tail) {
    // The tensor-core kernel multiplies whole key tiles: weight zero times whatever lies behind the
    // chunk's end must be zero, so the V rows up to the end of that tile are cleared (rows behind a
    // sequence's end belong to nobody).
    for (unsigned w = first; w < (unsigned)p.seqs.n * kExtTileKeys * pieces; w += stride) {
      const unsigned rx = w / pieces, piece = w - rx * pieces;
      const int s = (int)(rx / kExtTileKeys), x = (int)(rx % kExtTileKeys);
      const int b = p.seqs.b0 + s, t = p.seqs.tok0[s + 1] - p.seqs.tok0[s];
      const int end = p.len[b] + t, row = end + x;
      if (t == 0 || row >= p.cap || row >= (end + kExtTileKeys - 1) / kExtTileKeys * kExtTileKeys) continue;
      *reinterpret_cast<uint4*>(static_cast<T*>(p.V) + (((slab0 + b) * p.Hkv + h) * p.cap + row) * p.d + piece * E) = make_uint4(0u, 0u, 0u, 0u);
    }
  }
  if (p.publish) {
    // every CTA has read the lengths before it takes its ticket; the last one advances them
    __syncthreads();
    __shared__ int last;
    if (threadIdx.x == 0) last = atomicAdd(p.ticket, 1u) == gridDim.x * gridDim.y - 1;
    __syncthreads();
    if (last) {
      for (int s = threadIdx.x; s < p.seqs.n; s += blockDim.x) {
        const int b = p.seqs.b0 + s, t = p.seqs.tok0[s + 1] - p.seqs.tok0[s];
        if (t > 0 && p.len[b] + t <= p.cap) {
          p.len[b] += t;
          p.tot[b] += t;
          p.active[b] = 1;
        }
      }
      if (threadIdx.x == 0) *p.ticket = 0u;
    }
  }
}

// Advances the lengths by the accepted part of a staged chunk.  One block; tok0 holds the running sums.
__global__ void __launch_bounds__(kExtSeqs) extend_commit_kernel(const ExtendSeqs q, int* len, int* tot, int* active, int cap, int* err) {
  const int s = threadIdx.x;
  if (s >= q.n) return;
  const int t = q.tok0[s + 1] - q.tok0[s], b = q.b0 + s;
  if (t == 0) return;
  if (len[b] + t > cap) {
    atomicOr(err, kErrLenOverflow);
    return;
  }
  len[b] += t;
  tot[b] += t;
  active[b] = 1;
}

// A logit in base-2 units (before the visibility test), from the raw dot product.
__device__ __forceinline__ float ext_logit_exact(const ExtendParams& p, float dot, float slope, int apart) {
  float x = dot * p.scale;
  if (p.cap_logit > 0.f) x = p.cap_logit * tanhf(x / p.cap_logit);
  x -= slope * (float)apart;
  return x * 1.4426950408889634f;
}

template <typename T, bool KV8>
__device__ __forceinline__ float ext_row_value(const void* base, size_t idx, float scale) {
  if constexpr (KV8) return e4m3_to_float(static_cast<const uint8_t*>(base)[idx]) * scale;
  else return to_float(static_cast<const T*>(base)[idx]);
}

// Four adjoining elements (head sizes are multiples of 8, token strides of 16 bytes).
template <typename T, bool KV8>
__device__ __forceinline__ float4 ext_row_value4(const void* base, size_t idx, float scale) {
  if constexpr (KV8) {
    const uint32_t c = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(base) + idx);
    return make_float4(e4m3_to_float((uint8_t)c) * scale, e4m3_to_float((uint8_t)(c >> 8)) * scale, e4m3_to_float((uint8_t)(c >> 16)) * scale,
                       e4m3_to_float((uint8_t)(c >> 24)) * scale);
  } else if constexpr (sizeof(T) == 4) {
    return *reinterpret_cast<const float4*>(static_cast<const T*>(base) + idx);
  } else {
    const uint2 y = *reinterpret_cast<const uint2*>(static_cast<const T*>(base) + idx);
    return make_float4(__uint_as_float(y.x << 16), __uint_as_float(y.x & 0xffff0000u), __uint_as_float(y.y << 16), __uint_as_float(y.y & 0xffff0000u));
  }
}

__device__ __forceinline__ float ext_peer_float(const float* mine, int rank) {  // the same word of another CTA of the cluster
  uint32_t at;
  float x;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(at) : "memory");
  return x;
}

constexpr int kExtWarps = kExtGenericThreads / 32;
constexpr int kExtRowsPerWarp = kExtGenericRows / kExtWarps;
static_assert(kExtRowsPerWarp == 4 && kExtGenericKeys == 32, "a lane's registers");

constexpr size_t ext_generic_smem(int d) {  // Q [32][d], K [32][d + 4], V [32][d], a warp's weights [32][4], positions of the tile
  return ((size_t)kExtGenericRows * d + (size_t)kExtGenericKeys * (d + 4) + (size_t)kExtGenericKeys * d + (size_t)kExtGenericRows * kExtGenericKeys +
          kExtGenericKeys) * sizeof(float);
}

// Any type, any head size: fp32 FMA.  A work item = 32 query rows of one (layer, sequence, KV head), four per warp; lane =
// key for the products and the softmax, lane = column of head_dim for the output.  The weights are exact fp32 (exp2f,
// tanhf).  It serves fp32 slabs (where the tensor cores' formats could not hold 2e-5) and head sizes other than 128.
// Bound by FMA and shared-memory issue where there are many items; where they are few, by the chain of a tile's
// steps, so the key tiles of an item are dealt to a cluster of up to eight CTAs, which join their parts through
// one another's shared memory, in the order of their ranks (fp32, head_dim 64, 48 tokens behind 131 rows, six items:
// 44 us with a CTA per item, 11 to 12 us with clusters, the storing kernel included).
template <typename T, bool KV8>
__global__ void __launch_bounds__(kExtGenericThreads) extend_generic_kernel(const __grid_constant__ ExtendParams p, int cluster) {
  extern __shared__ __align__(16) float ext_sm[];
  const int d = p.d, ldk = d + 4, pieces = d / 4;
  float* sQ = ext_sm;
  float* sK = sQ + kExtGenericRows * d;
  float* sV = sK + kExtGenericKeys * ldk;
  float* sW = sV + kExtGenericKeys * d;
  int* sP = reinterpret_cast<int*>(sW + kExtGenericRows * kExtGenericKeys);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int item = (int)blockIdx.x / cluster, rank = (int)blockIdx.x - item * cluster;
  const unsigned piece_inv = 65536u / (unsigned)pieces + 1u;  // x / pieces = (x * piece_inv) >> 16 for x < 256 and up to 64 pieces
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int s = ext_find(p.seqs.item0, p.seqs.n, item);
  const ExtSeq e = ext_seq(p, s);
  if (!e.ok) return;  // (the whole cluster)
  const int layer = blockIdx.y / p.Hkv, h = blockIdx.y % p.Hkv;
  const int r0 = (item - p.seqs.item0[s]) * kExtGenericRows;
  const int rows = min(kExtGenericRows, e.t * p.G - r0);
  const size_t tok_base = (size_t)layer * p.total + p.seqs.tok0[s];
  const size_t slab = ((size_t)(p.layer0 + layer) * p.Nb + e.b) * p.Hkv + h;
  for (int x = lane; x < kExtRowsPerWarp * pieces; x += 32) {  // a warp stages its own four rows
    const int rl = (int)(((unsigned)x * piece_inv) >> 16), r = warp * kExtRowsPerWarp + rl, c = 4 * (x - rl * pieces);
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
    if (r < rows) {
      const int i = (r0 + r) / p.G, g = (r0 + r) - i * p.G;
      y = ext_row_value4<T, false>(p.q, (tok_base + i) * p.q_stride + (size_t)(h * p.G + g) * d + c, 1.f);
    }
    *reinterpret_cast<float4*>(sQ + r * d + c) = y;
  }
  // this warp's rows
  int tok[4];
  float slope[4], m[4], l[4], acc[4][8];  // l: this lane's part of the row's sum
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int r = r0 + warp * 4 + u;
    tok[u] = min(r / p.G, e.t - 1);
    slope[u] = p.slopes ? p.slopes[h * p.G + r % p.G] : 0.f;
    m[u] = -CUDART_INF_F;
    l[u] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[u][c] = 0.f;
  }
  const int prefix = p.seqs.prefix[s];
  const int i0 = r0 / p.G, i1 = min(e.t - 1, (r0 + rows - 1) / p.G);
  const int end = e.n + max(i1 + 1, prefix);
  // (positions ascend with the rows, so a row more than `window` rows back is more than `window` positions back)
  const int begin = p.window > 0 ? max(0, e.n + i0 - p.window + 1) : 0;
  for (int k0 = (begin / kExtGenericKeys + rank) * kExtGenericKeys; k0 < end; k0 += kExtGenericKeys * cluster) {
    __syncthreads();
#pragma unroll 2
    for (int x = lane; x < 4 * pieces; x += 32) {  // a warp stages four rows of K and of V
      const int rl = (int)(((unsigned)x * piece_inv) >> 16), r = warp * 4 + rl, c = 4 * (x - rl * pieces);
      const bool in = k0 + r < e.n + e.t;
      const size_t idx = (slab * p.cap + k0 + r) * d + c;
      float4 kk = make_float4(0.f, 0.f, 0.f, 0.f), vv = kk;
      if (in) {
        kk = ext_row_value4<T, KV8>(p.K, idx, 1.f);  // (k_scale is part of p.scale)
        vv = ext_row_value4<T, KV8>(p.V, idx, p.v_scale);
      }
      *reinterpret_cast<float4*>(sK + r * ldk + c) = kk;
      *reinterpret_cast<float4*>(sV + r * d + c) = vv;
    }
    if (tid < kExtGenericKeys) sP[tid] = k0 + tid < e.n + e.t ? p.pos[slab * p.cap + k0 + tid] : 0;
    __syncthreads();
    float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int c = 0; c < d; c += 4) {
      const float4 kv = *reinterpret_cast<const float4*>(sK + lane * ldk + c);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4 qv = *reinterpret_cast<const float4*>(sQ + (warp * 4 + u) * d + c);
        dot[u] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, dot[u]))));
      }
    }
    const int j = k0 + lane;
    float w[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int apart = abs(e.tot + tok[u] - sP[lane]);
      const bool visible = j < e.n + max(tok[u] + 1, prefix) && (p.window == 0 || apart < p.window);
      const float x = visible ? ext_logit_exact(p, dot[u], slope[u], apart) : -CUDART_INF_F;
      float mx = x;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float m_new = fmaxf(m[u], mx);
      const float alpha = m[u] == -CUDART_INF_F ? 0.f : exp2f(m[u] - m_new);
      // (all seen so far may be logits of -inf: they weigh nothing if any other follows, and leave 0 / 0 if none does)
      w[u] = visible ? exp2f(x - (m_new == -CUDART_INF_F ? 0.f : m_new)) : 0.f;
      l[u] = l[u] * alpha + w[u];
      m[u] = m_new;
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[u][c] *= alpha;
    }
    float* ww = sW + warp * 4 * kExtGenericKeys;  // the warp's weights, four rows of a key side by side
    *reinterpret_cast<float4*>(ww + 4 * lane) = make_float4(w[0], w[1], w[2], w[3]);
    __syncwarp();
#pragma unroll 4
    for (int kk = 0; kk < kExtGenericKeys; ++kk) {
      const float4 w4 = *reinterpret_cast<const float4*>(ww + 4 * kk);
      const float wk[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        if (c * 32 >= d) break;
        const int col = c * 32 + lane;
        const float vv = col < d ? sV[kk * d + col] : 0.f;
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (wk[u] != 0.f) acc[u][c] = fmaf(wk[u], vv, acc[u][c]);  // (a hidden row contributes nothing, whatever it holds)
      }
    }
  }
#pragma unroll
  for (int u = 0; u < 4; ++u)
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l[u] += __shfl_xor_sync(0xffffffffu, l[u], o);
  auto write = [&](int r, int col, float y) {  // (col < d)
    const int i = r / p.G, head = h * p.G + r - i * p.G;
    from_float(static_cast<T*>(p.out) + ((tok_base + i) * p.Hq + head) * d + col, y);
  };
  if (cluster == 1) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int rl = warp * 4 + u;
      if (rl >= rows) continue;
#pragma unroll
      for (int c = 0; c < 8; ++c)
        if (c * 32 + lane < d) write(r0 + rl, c * 32 + lane, acc[u][c] / l[u]);
      if (p.lse && lane == 0) p.lse[ext_lse_index(p, layer, h, p.seqs.tok0[s]) + r0 + rl] = m[u] + log2f(l[u]);
    }
    return;
  }
  // The parts join: every CTA leaves its own in shared memory (over K and V), and the rows are dealt to the cluster's warps.
  float* sA = sK;                              // [32][d]
  float* sML = sK + kExtGenericRows * d;       // [2][32]: maxima, sums
  __syncthreads();
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const int rl = warp * 4 + u;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      if (c * 32 + lane < d) sA[rl * d + c * 32 + lane] = acc[u][c];
    if (lane == 0) {
      sML[rl] = m[u];
      sML[kExtGenericRows + rl] = l[u];
    }
  }
  cluster_arrive();
  cluster_wait();
  for (int rl = rank * kExtWarps + warp; rl < rows; rl += cluster * kExtWarps) {
    const float pm = lane < cluster ? ext_peer_float(sML + rl, lane) : -CUDART_INF_F;
    const float pl = lane < cluster ? ext_peer_float(sML + kExtGenericRows + rl, lane) : 0.f;
    float M = pm;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));  // (clusters of up to eight)
    M = __shfl_sync(0xffffffffu, M, 0);
    const float f = pm == -CUDART_INF_F ? 0.f : exp2f(pm - M);
    float sum = pl * f;
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    sum = __shfl_sync(0xffffffffu, sum, 0);
    float fs[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) fs[k] = __shfl_sync(0xffffffffu, f, k);
    for (int col = lane; col < d; col += 32) {
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = k < cluster ? ext_peer_float(sA + rl * d + col, k) : 0.f;
      float o = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (fs[k] != 0.f) o = fmaf(fs[k], y[k], o);
      write(r0 + rl, col, o / sum);
    }
    if (p.lse && lane == 0) p.lse[ext_lse_index(p, layer, h, p.seqs.tok0[s]) + r0 + rl] = M + log2f(sum);
  }
  cluster_arrive();  // (no CTA ends while another reads from it)
  cluster_wait();
}

// What the mass kernels do with a row's total: exactly one thread owns the row.
__device__ __forceinline__ void ext_emit_mass(const ExtendParams& p, size_t row, float x) {
  if (p.mass) p.mass[row] = x;
  if (p.accumulate) {
    float sc = p.score[row], c = p.comp[row];
    kahan_add(sc, c, x);
    p.score[row] = sc;
    p.comp[row] = c;
  }
}

constexpr size_t ext_generic_mass_smem(int d) {  // K [32][d + 4], four query rows per warp, partial sums
  return ((size_t)kExtGenericKeys * (d + 4) + (size_t)kExtGenericRows * d + (size_t)kExtWarps * kExtGenericKeys) * sizeof(float);
}

// mass_j = sum over the chunk's tokens and the group's heads of the weight of row j, from the logits and each query
// row's log-sum-exp.  CTA = 32 rows of one slab; the warps take the query rows in turn, four at once (one read of
// K for four products), lane = key; the eight partial sums are added in a fixed order.
template <typename T, bool KV8>
__global__ void __launch_bounds__(kExtGenericThreads) extend_generic_mass_kernel(const __grid_constant__ ExtendParams p) {
  extern __shared__ __align__(16) float ext_sm[];
  const int d = p.d, ldk = d + 4, pieces = d / 4;
  float* sK = ext_sm;
  float* sQ = sK + kExtGenericKeys * ldk;
  float* sS = sQ + kExtGenericRows * d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const unsigned piece_inv = 65536u / (unsigned)pieces + 1u;  // x / pieces = (x * piece_inv) >> 16 for x < 256 and up to 64 pieces
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int layer = blockIdx.y / p.Hkv, h = blockIdx.y % p.Hkv, s = blockIdx.z;
  const ExtSeq e = ext_seq(p, s);
  const int k0 = blockIdx.x * kExtGenericKeys;
  if (!e.ok || e.t == 0 || k0 >= e.n + e.t) return;
  const size_t tok_base = (size_t)layer * p.total + p.seqs.tok0[s];
  const size_t slab = ((size_t)(p.layer0 + layer) * p.Nb + e.b) * p.Hkv + h;
  const float* lse = p.lse + ext_lse_index(p, layer, h, p.seqs.tok0[s]);
#pragma unroll 2
  for (int x = lane; x < 4 * pieces; x += 32) {  // a warp stages four rows of K
    const int rl = (int)(((unsigned)x * piece_inv) >> 16), r = warp * 4 + rl, c = 4 * (x - rl * pieces);
    *reinterpret_cast<float4*>(sK + r * ldk + c) =
        k0 + r < e.n + e.t ? ext_row_value4<T, KV8>(p.K, (slab * p.cap + k0 + r) * d + c, 1.f) : make_float4(0.f, 0.f, 0.f, 0.f);
  }
  __syncthreads();
  const int j = k0 + lane;
  const int pj = j < e.n + e.t ? p.pos[slab * p.cap + j] : 0;
  const int prefix = p.seqs.prefix[s], all = e.t * p.G;
  // (a token that sees row j: i >= j - n, or any where j lies before n + prefix)
  const int first = e.n + prefix > k0 ? 0 : max(0, k0 - e.n) * p.G;
  float* q4 = sQ + warp * 4 * d;
  float sum = 0.f;
  for (int r = first + 4 * warp; r < all; r += kExtGenericRows) {
    __syncwarp();
#pragma unroll 2
    for (int x = lane; x < 4 * pieces; x += 32) {
      const int rl = (int)(((unsigned)x * piece_inv) >> 16), c = 4 * (x - rl * pieces), row = min(r + rl, all - 1), i = row / p.G;
      *reinterpret_cast<float4*>(q4 + rl * d + c) =
          ext_row_value4<T, false>(p.q, (tok_base + i) * p.q_stride + (size_t)(h * p.G + row - i * p.G) * d + c, 1.f);
    }
    __syncwarp();
    float dot[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int c = 0; c < d; c += 4) {
      const float4 kv = *reinterpret_cast<const float4*>(sK + lane * ldk + c);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const float4 qv = *reinterpret_cast<const float4*>(q4 + u * d + c);
        dot[u] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, fmaf(qv.z, kv.z, fmaf(qv.w, kv.w, dot[u]))));
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (r + u >= all) break;
      const int i = (r + u) / p.G, head = h * p.G + r + u - i * p.G;
      const int apart = abs(e.tot + i - pj);
      if (j < e.n + max(i + 1, prefix) && (p.window == 0 || apart < p.window))
        sum += exp2f(ext_logit_exact(p, dot[u], p.slopes ? p.slopes[head] : 0.f, apart) - lse[r + u]);
    }
  }
  sS[warp * kExtGenericKeys + lane] = sum;
  __syncthreads();
  if (warp == 0 && j < e.n + e.t) {
    float x = 0.f;
#pragma unroll
    for (int w = 0; w < kExtWarps; ++w) x += sS[w * kExtGenericKeys + lane];
    ext_emit_mass(p, slab * p.cap + j, x);
  }
}

}  // namespace dynts
