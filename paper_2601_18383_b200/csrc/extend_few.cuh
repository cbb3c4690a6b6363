// The chunk operators for few query rows (definitions in extend.cuh): at most 128 rows (tokens times heads of the group) per
// sequence and KV head, head_dim 128, bf16 or 8-bit rows, no mass wanted: one token per sequence, drafted tokens,
// small trees.
//
// One launch.  A cluster of CTAs takes a slab's rows, in tiles of 32 dealt in equal runs, for up to 64 query rows; where slabs are few, clusters of
// their own take 32 query rows each (every one stores the chunk's rows, the same bits, so that it finds its own).  What the storing kernel does for the others
// (the chunk's rows into the slab, positions, scores, lengths) happens here: the CTA whose run holds a row of the chunk
// takes it from the caller's tensors into its tile in shared memory, and stores it.  The parts of a row meet
// in shared memory, the CTAs' through the cluster's.  (As three kernels, with the tensor-core kernel between, a tree of
// 12 behind 2048 rows took 25 us: the launches, their reads of lengths and plans, and a tile of 128 rows whose chain is the same
// for 48.)
//
// Inside a CTA a warp streams the tiles by TMA into a ring, as in the streaming decode kernel, and the consumer warps take 16 rows of
// K and V against 8 or 16 query rows each by mma.sync: products are few here (4 d flops per row, byte for byte 32 R / 128
// per byte of K and V), and M = 16 rows of K fit any number of query rows without the padding to 128 that tcgen05 asks for.
//   S[key][query] = K Q^T     16 keys on M, 8 queries on N, operands by ldmatrix from the swizzled tile, Q in registers
//   O^T[d][query] += V^T P    16 columns of head_dim on M; P through movmatrix
// Bound by HBM for long caches and many sequences, by the latency of launch, tile and exchange for few.
//
// A wave of CTAs takes 6 to 11 us whatever it reads (lengths, ring, exchange), so batches whose slabs need many waves go by the other kernels (the
// rule is at the launch).
//
// A weight of zero times a value that is not finite is not a number: V rows behind the chunk's end are zeroed in the
// tile, and an output row that is not finite is computed again by its warp from the rows it sees.
#pragma once

#include <cuda.h>

#include "decode_stream.cuh"
#include "extend.cuh"

namespace dynts {

constexpr int kFewKeys = 32;          // rows of a tile
constexpr int kFewMaxRows = 128, kFewSplitRows = 32;
// Weights for 8-bit rows are f16, whose smallest normal number is 2^-14: they are held times 2^15, and so are their sums, so that a weight keeps
// its 11 bits down to 2^-29 of the largest (many small ones beside a first token that takes most of the weight and has a small value).
constexpr float kFewF16Shift = 15.f;

// NB: blocks of 8 query rows per warp; RG: warps that share a run of keys; KA: groups of 2 RG warps that take the tiles in turn; PS: CTAs per SM.
// One token of 64 sequences, 512 slabs of 1028 rows, four CTAs per SM with two tiles each in flight 49 us, three with four tiles 60 (what does
// not fit at once comes after the rest); 8 slabs of 2048 rows in clusters of 8 the other way round, 11.7 and 10.1.
template <bool KV8, int NB, int RG, int KA, int PS>
struct FewShape {
  static constexpr int kRows = 8 * NB * RG;
  static constexpr int kWarps = 2 * RG * KA;              // consumers
  static constexpr int kThreads = 32 * (kWarps + 1);
  static constexpr int kTileBytes = kFewKeys * 2 * (KV8 ? 128 : 256);
  static constexpr int kPartBytes = kWarps * 8 * NB * 128 * 4;  // over the ring, when it is done
  static constexpr int kPerSm = PS;
  static constexpr int kStages = PS == 1 ? (KV8 ? 20 : 10) : PS == 2 ? (KV8 ? 12 : 6) : PS == 3 ? (KV8 ? 8 : 4) : (KV8 ? 6 : 2);
  static_assert(kStages % KA == 0 && kStages * kTileBytes >= kPartBytes, "a stage is always the same group's, and the parts fit the ring");
  static constexpr int kMlFloats = 2 * kWarps * 8 * NB;   // a warp's maxima and sums
  static constexpr size_t kSmem = (size_t)kStages * kTileBytes + 1024 + kMlFloats * 4 + kRows * 16 + 2 * kStages * 8 + 64;
};

struct FewParams {
  ExtendParams x;
  int cluster;
  float scale_log2;   // log2(e) * scale
  float cap_log2;     // c log2(e), or 0
  float cap_arg;      // 2 log2(e) scale / c
  float cap_y;        // scale / c
  float out_scale;    // v_scale for 8-bit rows
  unsigned int wait_limit;
};

__device__ __forceinline__ float4 few_peer4(uint32_t at, int rank) {  // 16 bytes of another CTA's shared memory
  uint32_t a;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float few_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float few_peer(uint32_t at, int rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// A query row again by a whole warp, exactly and from the rows it sees alone: a lane per key, then a lane per four columns.
template <bool KV8>
__device__ __noinline__ float4 few_row_again(const ExtendParams& x, int s, int layer, int h, int row, int n, int tot, int t) {
  const int lane = threadIdx.x & 31, i = row / x.G, g = row - i * x.G, tok0 = x.seqs.tok0[s];
  const size_t slab = ((size_t)(x.layer0 + layer) * x.Nb + x.seqs.b0 + s) * x.Hkv + h;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(x.q) + ((size_t)layer * x.total + tok0 + i) * x.q_stride + (size_t)(h * x.G + g) * 128;
  const ExtNode node = ext_node(x, tok0, i, t);
  const float slope = x.slopes ? x.slopes[h * x.G + g] : 0.f;
  const int end = n + max(i + 1, x.seqs.prefix[s]);
  const ExtTiles tiles = ext_tiles(x.window, x.sinks, x.tree != nullptr, n, 0, kFewKeys);
  auto logit = [&](int j, bool& visible) {
    visible = false;
    if (j >= end) return 0.f;
    const int pos = x.pos[slab * x.cap + j], apart = abs(tot + node.depth - pos);
    if (!ext_in_window(x, apart, pos) || !ext_below(node.order, ext_node(x, tok0, j - n, t))) return 0.f;
    visible = true;
    float dot = 0.f;
#pragma unroll 2
    for (int e = 0; e < 128; e += 4) {
      const uint2 qq = *reinterpret_cast<const uint2*>(q + e);
      const float4 k = ext_row_value4<__nv_bfloat16, KV8>(x.K, (slab * x.cap + j) * 128 + e, 1.f);
      dot = fmaf(__uint_as_float(qq.x << 16), k.x, dot);
      dot = fmaf(__uint_as_float(qq.x & 0xffff0000u), k.y, dot);
      dot = fmaf(__uint_as_float(qq.y << 16), k.z, dot);
      dot = fmaf(__uint_as_float(qq.y & 0xffff0000u), k.w, dot);
    }
    return ext_logit_exact(x, dot, slope, apart);
  };
  float m = -CUDART_INF_F, l = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int v = 0;; ++v) {
    const int k0 = ext_tile_of(v, tiles.sinks, tiles.jump) * kFewKeys;
    if (k0 >= end) break;
    bool visible;
    const float y = logit(k0 + lane, visible);
    float mx = visible ? y : -CUDART_INF_F;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float mn = fmaxf(m, mx), keep = m == -CUDART_INF_F ? 0.f : exp2f(m - mn);
    const float w = visible ? exp2f(y - (mn == -CUDART_INF_F ? 0.f : mn)) : 0.f;
    m = mn;
    l = l * keep + w;
    acc = make_float4(acc.x * keep, acc.y * keep, acc.z * keep, acc.w * keep);
    for (unsigned some = __ballot_sync(0xffffffffu, w != 0.f); some; some &= some - 1) {
      const int kk = __ffs(some) - 1;
      const float wk = __shfl_sync(0xffffffffu, w, kk);
      const float4 vv = ext_row_value4<__nv_bfloat16, KV8>(x.V, (slab * x.cap + k0 + kk) * 128 + 4 * lane, 1.f);
      acc = make_float4(fmaf(wk, vv.x, acc.x), fmaf(wk, vv.y, acc.y), fmaf(wk, vv.z, acc.z), fmaf(wk, vv.w, acc.w));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
  return make_float4(acc.x / l, acc.y / l, acc.z / l, acc.w / l);
}

template <bool KV8, bool MODS, int NB, int RG, int KA, int PS>
__global__ void __launch_bounds__((FewShape<KV8, NB, RG, KA, PS>::kThreads), (FewShape<KV8, NB, RG, KA, PS>::kPerSm))
extend_few_kernel(const __grid_constant__ FewParams p, const __grid_constant__ CUtensorMap map) {
  using S = FewShape<KV8, NB, RG, KA, PS>;
  constexpr int NS = S::kStages;
  extern __shared__ __align__(1024) uint8_t few_raw[];
  uint8_t* ring = few_raw + ((1024u - (smem_u32(few_raw) & 1023u)) & 1023u);
  float* s_ml = reinterpret_cast<float*>(ring + NS * S::kTileBytes);   // [warps][2][8 NB]
  int4* s_row = reinterpret_cast<int4*>(s_ml + S::kMlFloats);          // end of what the row sees, position, order, slope
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_row + S::kRows);      // full, empty
  volatile int* s_abort = reinterpret_cast<volatile int*>(bars + 2 * NS);
  const uint32_t bar_full = smem_u32(bars), bar_empty = bar_full + 8 * NS;
  const ExtendParams& x = p.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int s = (int)blockIdx.x / p.cluster, rank = (int)blockIdx.x - s * p.cluster;
  const int layer = (int)blockIdx.y / x.Hkv, h = (int)blockIdx.y - layer * x.Hkv;
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(bar_full + 8 * i, 1);
      mbar_init(bar_empty + 8 * i, 2 * RG);
    }
    *s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&map)) : "memory");
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = x.seqs.b0 + s, tok0 = x.seqs.tok0[s], t = x.seqs.tok0[s + 1] - tok0, prefix = x.seqs.prefix[s];
  const int q0 = (int)blockIdx.z * S::kRows;  // this cluster's query rows, from here on
  const int n = x.len[b], tot = x.tot[b], all_rows = t * x.G, rows = min(S::kRows, all_rows - q0);
  const bool fits = n >= 0 && n + t <= x.cap, work = rows > 0 && fits;  // (the same in the whole cluster)
  if (t > 0 && !fits && tid == 0 && rank == 0) atomicOr(x.err, kErrLenOverflow);
  const size_t slab = ((size_t)(x.layer0 + layer) * x.Nb + b) * x.Hkv + h;
  const ExtTiles tiles = ext_tiles(x.window, x.sinks, x.tree != nullptr, n, 0, kFewKeys);
  const int all = work ? (n + t + kFewKeys - 1) / kFewKeys - tiles.jump : 0;
  const int v0 = (int)((long long)all * rank / p.cluster), v1 = (int)((long long)all * (rank + 1) / p.cluster);
  if (tid < S::kRows) {
    int4 w = make_int4(0, 0, 0, 0);
    if (work && tid < rows) {
      const int i = (q0 + tid) / x.G;
      const ExtNode node = ext_node(x, tok0, i, t);
      w = make_int4(n + max(i + 1, prefix), tot + node.depth, node.order, x.slopes ? __float_as_int(x.slopes[h * x.G + q0 + tid - i * x.G] * 1.4426950408889634f) : 0);
    }
    s_row[tid] = w;
  }
  __syncthreads();

  if (warp == S::kWarps) {
    // ================= the warp that loads: a tile of K and V per stage =================
    const uint64_t policy = l2_evict_first_policy();
    for (int v = v0; v < v1 && !*s_abort; ++v) {
      const int it = v - v0, st = it % NS;
      if (it >= NS) mbar_wait(bar_empty + 8 * st, (uint32_t)((it / NS - 1) & 1), s_abort, x.err, p.wait_limit);
      __syncwarp();
      if (*s_abort) break;
      if (lane == 0) {
        const int row = (int)(slab * x.cap) + ext_tile_of(v, tiles.sinks, tiles.jump) * kFewKeys;
        const uint32_t dst = smem_u32(ring) + (uint32_t)st * S::kTileBytes, bb = bar_full + 8 * st;
        mbar_arrive_expect_tx(bb, S::kTileBytes);
        tma_load_3d(dst, &map, 0, row, 0, bb, policy);  // K and V boxes of 32 rows; 16-bit rows: a half of head_dim each time
        if constexpr (!KV8) tma_load_3d(dst + 2 * kStBoxBytes, &map, 64, row, 0, bb, policy);
      }
      __syncwarp();
    }
    if (*s_abort && lane == 0)  // something gave up: a bounded time for the loads in flight
      for (int i = 0; i < NS; ++i)
        for (uint32_t ph = 0; ph < 2; ++ph)
          for (uint32_t w = 0; w < (1u << 14); ++w)
            if (mbar_try_wait(bar_full + 8 * i, ph)) break;
  } else if (v1 > v0) {
    // ================= the warps that compute: 16 rows of K and V against 8 NB query rows =================
    const int gid = lane >> 2, tig = lane & 3;
    const int rg = warp % RG, u16 = (warp / RG & 1) * 16, ga = warp / (2 * RG);
    const int lrow = u16 + ((lane >> 4) << 3) + (lane & 7), lchk = (lane >> 3) & 1;  // ldmatrix: row, 16-byte piece parity
    const int r0 = rg * 8 * NB;
    // Q fragments: rows r0 + 8 nb + gid, two pieces of a k-step (8-bit rows: in the order of a register of codes, as f16)
    uint32_t qa[NB][8][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = q0 + r0 + 8 * nb + gid, i = r / x.G;
      const uint32_t* hq = reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(x.q) + ((size_t)layer * x.total + tok0 + i) * x.q_stride +
                                                              (size_t)(h * x.G + r - i * x.G) * 128);
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) {
        if constexpr (KV8) {
          const uint2 w = r < all_rows ? *reinterpret_cast<const uint2*>(hq + 8 * kk + 2 * tig) : make_uint2(0u, 0u);
          qa[nb][kk][0] = bf16x2_to_half2(w.x);
          qa[nb][kk][1] = bf16x2_to_half2(w.y);
        } else {
          qa[nb][kk][0] = r < all_rows ? hq[8 * kk + tig] : 0u;
          qa[nb][kk][1] = r < all_rows ? hq[8 * kk + 4 + tig] : 0u;
        }
      }
    }
    float o[NB][8][4], m[NB][2], l[NB][2];  // queries 2 tig and 2 tig + 1 of each block
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int mb = 0; mb < 8; ++mb)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[nb][mb][e] = 0.f;
      m[nb][0] = m[nb][1] = -CUDART_INF_F;
      l[nb][0] = l[nb][1] = 0.f;
    }
    const bool placed = MODS && (x.window > 0 || x.slopes != nullptr);
#pragma unroll 1
    for (int it = ga; it < v1 - v0; it += KA) {
      const int st = it % NS, k0 = ext_tile_of(v0 + it, tiles.sinks, tiles.jump) * kFewKeys;
      const int j[2] = {k0 + u16 + gid, k0 + u16 + gid + 8};  // this thread's keys
      const bool fresh = k0 + kFewKeys > n;                   // the tile holds rows of the chunk, or ends behind it
      int pos[2] = {0, 0};
      if (placed) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (j[e] < n) pos[e] = x.pos[slab * x.cap + j[e]];
      }
      mbar_wait(bar_full + 8 * st, (uint32_t)((it / NS) & 1), s_abort, x.err, p.wait_limit);
      __syncwarp();
      uint8_t* tile = ring + (size_t)st * S::kTileBytes;
      if (fresh) {
        // the chunk's rows into the tile and the slab; V rows behind them are zero.  By the warps of the group, 16 bytes at a time.
        const int gt = (warp - ga * 2 * RG) * 32 + lane;
        constexpr int kPieces = KV8 ? 8 : 16;
        for (int w = gt; w < kFewKeys * 2 * kPieces; w += 64 * RG) {
          const int r = w / (2 * kPieces), y = w - r * 2 * kPieces, isv = y / kPieces, ch = y - isv * kPieces, i = k0 + r - n;
          if (i < 0 || (i >= t && !isv)) continue;
          uint8_t* at = KV8 ? tile + isv * kStBoxBytes + r * 128 + ((ch ^ (r & 7)) << 4) : tile + (isv + 2 * (ch >> 3)) * kStBoxBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4);
          uint4 val = make_uint4(0u, 0u, 0u, 0u);
          if (i < t) {
            const size_t src = (size_t)layer * x.total + tok0 + i;
            const __nv_bfloat16* from = static_cast<const __nv_bfloat16*>(isv ? x.v : x.k) + src * (isv ? x.v_stride : x.k_stride) + (size_t)h * 128 + ch * (128 / kPieces);
            if constexpr (KV8) {
              const uint4 a = reinterpret_cast<const uint4*>(from)[0], c = reinterpret_cast<const uint4*>(from)[1];
              const float sc = isv ? x.v_scale : x.k_scale;
              const uint32_t in[8] = {a.x, a.y, a.z, a.w, c.x, c.y, c.z, c.w};
              uint32_t o4[4];
#pragma unroll
              for (int e = 0; e < 4; ++e)
                o4[e] = (uint32_t)float2_to_e4m3x2(__fdiv_rn(__uint_as_float(in[2 * e] << 16), sc), __fdiv_rn(__uint_as_float(in[2 * e] & 0xffff0000u), sc)) |
                        ((uint32_t)float2_to_e4m3x2(__fdiv_rn(__uint_as_float(in[2 * e + 1] << 16), sc), __fdiv_rn(__uint_as_float(in[2 * e + 1] & 0xffff0000u), sc)) << 16);
              val = make_uint4(o4[0], o4[1], o4[2], o4[3]);
            } else {
              val = *reinterpret_cast<const uint4*>(from);
            }
            const size_t row = slab * x.cap + n + i;
            reinterpret_cast<uint4*>(static_cast<uint8_t*>(isv ? x.V : x.K) + row * (16 * kPieces))[ch] = val;
            if (y == 0) {
              x.pos[row] = tot + ext_node(x, tok0, i, t).depth;
              x.score[row] = x.s_new ? x.s_new[tok0 + i] : 0.f;
              x.comp[row] = 0.f;
            }
          }
          *reinterpret_cast<uint4*>(at) = val;
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // (the stage's next tile comes by TMA)
        asm volatile("bar.sync %0, %1;" ::"r"(2 + ga), "n"(64 * RG) : "memory");
      }
      // S = K Q^T (two accumulators, so that the chain of dependent products is half as long)
      float sc[NB][4];
      uint32_t fr[8][4];
      {
        float a0[NB][4], a1[NB][4];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) a0[nb][e] = a1[nb][e] = 0.f;
        const uint32_t kbase = smem_u32(tile) + lrow * 128, vbase = kbase + kStBoxBytes;
        if constexpr (KV8) {
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t k0r, k1r, k2r, k3r, f0, f1, f2, f3;
            ldmatrix_x4(kbase + (((2 * c + lchk) ^ (lrow & 7)) << 4), k0r, k1r, k2r, k3r);
            e4m3x4_to_half2x2(k0r, f0, f2);
            e4m3x4_to_half2x2(k2r, f1, f3);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_f16_m16n8k16(a0[nb], f0, f1, f2, f3, qa[nb][2 * c][0], qa[nb][2 * c][1]);
            e4m3x4_to_half2x2(k1r, f0, f2);
            e4m3x4_to_half2x2(k3r, f1, f3);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma_f16_m16n8k16(a1[nb], f0, f1, f2, f3, qa[nb][2 * c + 1][0], qa[nb][2 * c + 1][1]);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) ldmatrix_x4_trans(vbase + (((2 * c + lchk) ^ (lrow & 7)) << 4), fr[c][0], fr[c][1], fr[c][2], fr[c][3]);
        } else {
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            ldmatrix_x4(kbase + (kk >> 2) * (2 * kStBoxBytes) + (((((2 * kk) & 7) + lchk) ^ (lrow & 7)) << 4), fr[kk][0], fr[kk][1], fr[kk][2], fr[kk][3]);
#pragma unroll
          for (int kk = 0; kk < 8; kk += 2)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              mma_bf16_m16n8k16(a0[nb], fr[kk][0], fr[kk][2], fr[kk][1], fr[kk][3], qa[nb][kk][0], qa[nb][kk][1]);
              mma_bf16_m16n8k16(a1[nb], fr[kk + 1][0], fr[kk + 1][2], fr[kk + 1][1], fr[kk + 1][3], qa[nb][kk + 1][0], qa[nb][kk + 1][1]);
            }
#pragma unroll
          for (int mb = 0; mb < 8; ++mb)
            ldmatrix_x4_trans(vbase + (mb >> 2) * (2 * kStBoxBytes) + (((((2 * mb) & 7) + lchk) ^ (lrow & 7)) << 4), fr[mb][0], fr[mb][1], fr[mb][2], fr[mb][3]);
        }
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nb][e] = a0[nb][e] + a1[nb][e];  // [key gid | gid + 8][query 2 tig | 2 tig + 1]
      }
      // logits, in base-2 units; what is hidden is -inf
      if constexpr (MODS) {
        // c tanh(y), y = logit / c: by the polynomial, off by a rounding or two of the result, while every logit of the warp's tile lies below three
        // quarters of the cap; else as c - 2 c / (1 + e^(2 y)), off by a few 2^-24 of c (of logits far below the cap nothing would
        // be left).
        if (x.cap_logit > 0.f) {
          float top = 0.f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, fabsf(sc[nb][e]));
          if (__all_sync(0xffffffffu, top * p.cap_y <= 0.75f)) {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float y = sc[nb][e] * p.cap_y, z = y * y;
                float f = ext_cap_term(5);
#pragma unroll
                for (int i = 4; i >= 0; --i) f = fmaf(f, z, ext_cap_term(i));
                sc[nb][e] = f * y * p.cap_log2;
              }
          } else {
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e) sc[nb][e] = fmaf(-2.f * p.cap_log2, few_rcp(1.f + fast_exp2(sc[nb][e] * p.cap_arg)), p.cap_log2);
          }
        }
      }
      const float scale = MODS && x.cap_logit > 0.f ? 1.f : p.scale_log2;
      ExtNode node[2] = {{0, 0x7fffffff, 0}, {0, 0x7fffffff, 0}};
      if (fresh && MODS) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          node[e] = ext_node(x, tok0, j[e] - n, t);
          if (j[e] >= n) pos[e] = tot + node[e].depth;
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if (!placed && !fresh) {  // all of it is seen by all
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[nb][e] *= scale;
          continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int4 row = s_row[r0 + 8 * nb + 2 * tig + (e & 1)];
          const int k = e >> 1;
          float z = sc[nb][e] * scale;
          bool seen = j[k] < row.x;
          if constexpr (MODS) {
            const int apart = abs(row.y - pos[k]);
            z -= __int_as_float(row.w) * (float)apart;
            seen = seen && ext_in_window(x, apart, pos[k]) && ext_below(row.z, node[k]);
          }
          sc[nb][e] = seen ? z : -CUDART_INF_F;
        }
      }
      // online softmax over the 16 keys, and the weights as the second product's operand
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float u[2] = {fmaxf(sc[nb][0], sc[nb][2]), fmaxf(sc[nb][1], sc[nb][3])}, keep[2], safe[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
#pragma unroll
          for (int o_ = 4; o_ < 32; o_ <<= 1) u[q] = fmaxf(u[q], __shfl_xor_sync(0xffffffffu, u[q], o_));
          const float mn = fmaxf(m[nb][q], u[q]);
          const float base = mn == -CUDART_INF_F ? 0.f : mn;
          keep[q] = m[nb][q] == mn ? 1.f : fast_exp2(m[nb][q] - base);  // (also while the row has seen nothing)
          safe[q] = KV8 ? base - kFewF16Shift : base;
          m[nb][q] = mn;
        }
        const float w0 = fast_exp2(sc[nb][0] - safe[0]), w1 = fast_exp2(sc[nb][1] - safe[1]), w2 = fast_exp2(sc[nb][2] - safe[0]), w3 = fast_exp2(sc[nb][3] - safe[1]);
        l[nb][0] = l[nb][0] * keep[0] + (w0 + w2);
        l[nb][1] = l[nb][1] * keep[1] + (w1 + w3);
        const uint32_t pb0 = movmatrix_trans(KV8 ? pack_half2(w0, w1) : pack_bf16x2(w0, w1)), pb1 = movmatrix_trans(KV8 ? pack_half2(w2, w3) : pack_bf16x2(w2, w3));
        if (!__all_sync(0xffffffffu, keep[0] == 1.f && keep[1] == 1.f)) {
#pragma unroll
          for (int mb = 0; mb < 8; ++mb) {
            o[nb][mb][0] *= keep[0];
            o[nb][mb][1] *= keep[1];
            o[nb][mb][2] *= keep[0];
            o[nb][mb][3] *= keep[1];
          }
        }
#pragma unroll
        for (int mb = 0; mb < 8; ++mb) {
          if constexpr (KV8) {
            uint32_t a0, a1, a2, a3;  // -> (key, key + 1) pairs of columns 2 gid and 2 gid + 1
            e4m3x4_to_half2x2(__byte_perm(fr[mb >> 1][mb & 1], 0u, 0x3120), a0, a1);
            e4m3x4_to_half2x2(__byte_perm(fr[mb >> 1][2 + (mb & 1)], 0u, 0x3120), a2, a3);
            mma_f16_m16n8k16(o[nb][mb], a0, a1, a2, a3, pb0, pb1);
          } else {
            mma_bf16_m16n8k16(o[nb][mb], fr[mb][0], fr[mb][1], fr[mb][2], fr[mb][3], pb0, pb1);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar_empty + 8 * st);
    }
    // this warp's part, over the ring once every warp is done with it
    asm volatile("bar.sync 1, %0;" ::"n"(32 * S::kWarps) : "memory");
    float* part = reinterpret_cast<float*>(ring) + (size_t)warp * (8 * NB * 128);
    float* ml = s_ml + warp * 16 * NB;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        float y = l[nb][q];
#pragma unroll
        for (int o_ = 4; o_ < 32; o_ <<= 1) y += __shfl_xor_sync(0xffffffffu, y, o_);
        const int r = 8 * nb + 2 * tig + q;
        if (gid == 0) {
          ml[r] = m[nb][q];
          ml[8 * NB + r] = y;
        }
#pragma unroll
        for (int mb = 0; mb < 8; ++mb) {  // (columns 16 mb + gid and + 8; 8-bit rows: 16 mb + 2 gid and + 1)
          part[r * 128 + 16 * mb + (KV8 ? 2 * gid : gid)] = o[nb][mb][q];
          part[r * 128 + 16 * mb + (KV8 ? 2 * gid + 1 : gid + 8)] = o[nb][mb][2 + q];
        }
      }
    asm volatile("bar.sync 1, %0;" ::"n"(32 * S::kWarps) : "memory");
    // the CTA's: the warps of a row's block of queries, in order; left in the first one's place
    for (int r = warp; r < S::kRows; r += S::kWarps) {
      const int w0 = r / (8 * NB), rl = r - w0 * 8 * NB;
      float M = -CUDART_INF_F, L = 0.f;
#pragma unroll
      for (int k = 0; k < 2 * KA; ++k) M = fmaxf(M, s_ml[(w0 + RG * k) * 16 * NB + rl]);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 2 * KA; ++k) {
        const float* src = s_ml + (w0 + RG * k) * 16 * NB;
        const float f = src[rl] == -CUDART_INF_F ? 0.f : fast_exp2(src[rl] - M);
        const float4 y = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(ring) + (size_t)(w0 + RG * k) * (8 * NB * 128) + rl * 128 + 4 * lane);
        L = fmaf(f, src[8 * NB + rl], L);
        acc = make_float4(fmaf(f, y.x, acc.x), fmaf(f, y.y, acc.y), fmaf(f, y.z, acc.z), fmaf(f, y.w, acc.w));
      }
      __syncwarp();
      *reinterpret_cast<float4*>(reinterpret_cast<float*>(ring) + (size_t)w0 * (8 * NB * 128) + rl * 128 + 4 * lane) = acc;
      if (lane == 0) {
        s_ml[w0 * 16 * NB + rl] = M;
        s_ml[w0 * 16 * NB + 8 * NB + rl] = L;
      }
    }
  } else {
    for (int r = tid; r < S::kRows; r += 32 * S::kWarps) {  // no key of this slab is this CTA's
      const int w0 = r / (8 * NB), rl = r - w0 * 8 * NB;
      s_ml[w0 * 16 * NB + rl] = -CUDART_INF_F;
      s_ml[w0 * 16 * NB + 8 * NB + rl] = 0.f;
    }
  }
  __syncthreads();
  if (p.cluster > 1) {
    cluster_arrive();
    cluster_wait();
  }
  if (work && warp < S::kWarps && !*s_abort) {
    // the cluster's parts of a row, in the order of the ranks; a row per warp
    for (int r = rank * S::kWarps + warp; r < rows; r += p.cluster * S::kWarps) {
      const int w0 = r / (8 * NB), rl = r - w0 * 8 * NB;
      const uint32_t at_ml = smem_u32(s_ml + w0 * 16 * NB + rl), at = smem_u32(ring) + (uint32_t)((w0 * 8 * NB + rl) * 128 + 4 * lane) * 4u;
      const float mk = lane < p.cluster ? few_peer(at_ml, lane) : -CUDART_INF_F, lk = lane < p.cluster ? few_peer(at_ml + 32u * NB, lane) : 0.f;
      float M = mk;
#pragma unroll
      for (int o_ = 16; o_ > 0; o_ >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o_));
      const float f = mk == -CUDART_INF_F ? 0.f : fast_exp2(mk - M);
      float L = f * lk;
#pragma unroll
      for (int o_ = 16; o_ > 0; o_ >>= 1) L += __shfl_xor_sync(0xffffffffu, L, o_);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int k = 0; k < p.cluster; ++k) {
        const float fk = __shfl_sync(0xffffffffu, f, k);
        if (fk == 0.f) continue;
        const float4 y = few_peer4(at, k);
        acc = make_float4(fmaf(fk, y.x, acc.x), fmaf(fk, y.y, acc.y), fmaf(fk, y.z, acc.z), fmaf(fk, y.w, acc.w));
      }
      const float inv = 1.f / L;
      acc = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
      const bool fine = (acc.x + acc.y) * 0.f == 0.f && (acc.z + acc.w) * 0.f == 0.f;
      if (!__all_sync(0xffffffffu, fine)) acc = few_row_again<KV8>(x, s, layer, h, q0 + r, n, tot, t);
      const int i = (q0 + r) / x.G;
      __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(x.out) + (((size_t)layer * x.total + tok0 + i) * x.Hq + h * x.G + q0 + r - i * x.G) * 128 + 4 * lane;
      *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(acc.x * p.out_scale, acc.y * p.out_scale), pack_bf16x2(acc.z * p.out_scale, acc.w * p.out_scale));
    }
  }
  if (x.publish) {
    // every CTA has read the lengths before it takes its ticket; the last one advances them
    __syncthreads();
    __shared__ int last;
    if (tid == 0) last = atomicAdd(x.ticket, 1u) == gridDim.x * gridDim.y * gridDim.z - 1;
    __syncthreads();
    if (last) {
      for (int q = tid; q < x.seqs.n; q += S::kThreads) {
        const int bq = x.seqs.b0 + q, tq = x.seqs.tok0[q + 1] - x.seqs.tok0[q];
        if (tq > 0 && x.len[bq] + tq <= x.cap) {
          x.len[bq] += tq;
          x.tot[bq] += tq;
          x.active[bq] = 1;
        }
      }
      if (tid == 0) *x.ticket = 0u;
    }
  }
  if (p.cluster > 1) {
    __syncwarp();
    cluster_arrive();  // (no CTA ends while another reads from it)
    cluster_wait();
  }
}

}  // namespace dynts
