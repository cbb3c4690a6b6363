// Tensor-core kernels of the chunk operators (definitions in extend.cuh) for head_dim 128, bf16 rows or
// 8-bit rows: tcgen05.mma with the accumulators in tensor memory.
//
// extend_tc_kernel.  A tile of 128 query rows packs the group's G heads of floor(128 / G) neighbouring
// tokens, so a row of K and V is read once for all of them whatever the chunk's length.  A work item =
// (tile of query rows, KV head, layer, sequence, part of the key rows): where the tiles alone do not fill
// the GPU (few tokens behind a long cache) the key rows of a tile are cut into parts that run side by
// side; each leaves its unnormalised output, maximum and sum in the scratch, and the last part to finish
// (a counter per tile) joins them in a fixed order.  Two CTAs per SM; per 64 keys
//     S  = Q K^T      M 128 x N 64 x K 128     operands from shared memory
//     P  = exp2(S * scale - max)               softmax warps, thread = query row = tensor-memory lane
//     O += P V        M 128 x N 128 x K 64     P from tensor memory
// The warps' roles, the double-buffered S, the lazy rescale and the barriers are those of the prompt
// attention (prefill_attn.cuh); what differs is where the rows come from, the items, and the row
// arithmetic, which knows caps, biases, windows and prefixes (MODS).  A warp whose 32 rows hold no
// query (a short chunk) skips the arithmetic.
//
// Rows of 16 bits arrive by TMA from the slabs.  8-bit rows (KV8) are read by two warps as codes, one
// tile ahead in registers, widened to f16 (exact) and stored into the same swizzled tiles; queries
// (an f16 copy made by the storing kernel) and weights are then f16 too.
//
// A weight of zero times a value that is not finite is not a number, and the MMA multiplies whole
// tiles: rows behind the chunk's end are zero (the storing kernel clears them, KV8 writes zeros), and an
// output element that is not finite is computed again by its warp from the visible rows alone.
#pragma once

#include <cuda.h>
#include <type_traits>

#include "extend.cuh"
#include "prefill_attn.cuh"
#include "tc5.cuh"

namespace dynts {

constexpr int kXtThreads = 256;
constexpr int kXtRows = 128;
constexpr int kXtPartFloats = 130;  // per query row of a part: 128 outputs, maximum, sum
constexpr int kXtSmemBytes = kPfQBytes + 4 * kPfKvBytes + kPfOutStageBytes + 128 + kExtSeqs * 4;

struct ExtendTcParams {
  ExtendParams x;       // seqs.item0: first (tile, part) pair of each sequence; heads and layers multiply it
  int parts[kExtSeqs];  // parts each tile's key rows are cut into
  int tokens_per_tile;  // floor(128 / G)
  int lh;               // n_layers * Hkv
  int n_work;           // items
  int part_rows;        // query rows a part's scratch has room for
  float* part;          // [n_work][128 / 4 + 1][part_rows] float4 / float2 pieces, or NULL: no tile is cut
  int* stop;
  float scale_log2;     // log2(e) * scale
  float cap_log2;       // c * log2(e)
  float cap_arg;        // 2 log2(e) * scale / c
};

struct XtCursor {
  int it, ord;            // position in this CTA's list; how many items came before
  int j, nkt, kt0;        // tile within the item, tiles of the item, first key tile
  int s, layer, h, lh, n; // sequence of the launch, layer, KV head; rows held
  int i0, rows;           // first token of the chunk, query rows
  int u0, split, n_split; // item index of the tile's first part; this part; parts that hold any keys
};

__device__ __forceinline__ void xt_seek(XtCursor& c, int it, int n_items, const ExtendTcParams& p, const int* s_n) {
  c.j = 0;
  for (; it < n_items; ++it) {
    const int slot = 2 * (int)blockIdx.x >= (int)gridDim.x ? n_items - 1 - it : it;
    const int w = (int)blockIdx.x + slot * (int)gridDim.x;
    const int u = w / p.lh;
    c.lh = w - u * p.lh;
    c.s = ext_find(p.x.seqs.item0, p.x.seqs.n, u);
    const int S = p.parts[c.s], first = p.x.seqs.item0[c.s];
    const int n_tiles = (p.x.seqs.item0[c.s + 1] - first) / S;
    const int qi = (u - first) / S;
    c.split = u - first - qi * S;
    c.u0 = u - c.split;
    c.n = s_n[c.s];
    if (c.n < 0) continue;  // no room for the chunk: nothing was stored
    const int t = p.x.seqs.tok0[c.s + 1] - p.x.seqs.tok0[c.s];
    c.i0 = (n_tiles - 1 - qi) * p.tokens_per_tile;  // heaviest first
    const int i1 = min(t, c.i0 + p.tokens_per_tile);
    c.rows = (i1 - c.i0) * p.x.G;
    const int end = c.n + max(i1, p.x.seqs.prefix[c.s]);
    // (positions ascend with the rows, so a row more than `window` rows back is more than `window` positions back)
    const int b = p.x.window > 0 ? max(0, c.n + c.i0 - p.x.window + 1) / kPfKeys : 0;
    const int total = (end + kPfKeys - 1) / kPfKeys - b;
    const int per = (total + S - 1) / S;
    c.n_split = (total + per - 1) / per;
    if (c.split >= c.n_split) continue;
    c.kt0 = b + c.split * per;
    c.nkt = min(per, total - c.split * per);
    c.layer = c.lh / p.x.Hkv;
    c.h = c.lh - c.layer * p.x.Hkv;
    break;
  }
  c.it = it;
}
__device__ __forceinline__ void xt_advance(XtCursor& c, int n_items, const ExtendTcParams& p, const int* s_n) {
  if (++c.j == c.nkt) {
    ++c.ord;
    xt_seek(c, c.it + 1, n_items, p, s_n);
  }
}

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// 64 rows of 128 codes, held by a warp as 16 pieces of 16 codes per lane (rows 4 i + lane / 8, piece lane % 8).
struct XtCodes {
  uint4 c[16];
};
__device__ __forceinline__ void xt_load_codes(XtCodes& r, const uint8_t* base, int key0, int end, int lane) {
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = key0 + 4 * i + (lane >> 3);
    r.c[i] = row < end ? ldg_stream(base + (size_t)row * 128 + (lane & 7) * 16) : make_uint4(0u, 0u, 0u, 0u);
  }
}
// ... widened into a tile [2 halves of head_dim][rows][128 B], 16-byte chunks swizzled by row.  The lanes of
// the second half write their two chunks in the other order, so that a store's eight lanes meet eight banks.
__device__ __forceinline__ void xt_store_codes(const XtCodes& r, uint8_t* tile, int half_bytes, int lane) {
  const int piece = lane & 7, half = piece >> 2;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int row = 4 * i + (lane >> 3);
    uint8_t* dst = tile + half * half_bytes + row * 128;
    const uint32_t w[4] = {r.c[i].x, r.c[i].y, r.c[i].z, r.c[i].w};
    uint4 y[2];
    uint32_t* o = reinterpret_cast<uint32_t*>(y);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      o[2 * u] = e4m3x2_to_half2((unsigned short)(w[u] & 0xffffu));
      o[2 * u + 1] = e4m3x2_to_half2((unsigned short)(w[u] >> 16));
    }
    const int c0 = 2 * (piece & 3);
    const uint4 a = half ? y[1] : y[0], b = half ? y[0] : y[1];
    const int ca = c0 + half, cb = c0 + 1 - half;
    *reinterpret_cast<uint4*>(dst + ((ca ^ (row & 7)) << 4)) = a;
    *reinterpret_cast<uint4*>(dst + ((cb ^ (row & 7)) << 4)) = b;
  }
}

// One query row again, by its whole warp, from the visible rows of [k0, k1) alone: sum of exp2(x_j - m) v_j,
// lane = four columns.  For rows whose output is not finite (a hidden row held something that is not).
template <bool KV8>
__device__ __noinline__ float4 xt_row_again(const ExtendTcParams& p, int s, int layer, int h, int n, int i, int g, int k0, int k1, float m) {
  const ExtendParams& x = p.x;
  const int lane = threadIdx.x & 31, b = x.seqs.b0 + s, t = x.seqs.tok0[s + 1] - x.seqs.tok0[s];
  const size_t slab = ((size_t)(x.layer0 + layer) * x.Nb + b) * x.Hkv + h;
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(x.q) + ((size_t)layer * x.total + x.seqs.tok0[s] + i) * x.q_stride + (size_t)(h * x.G + g) * 128;
  const int tot = x.tot[b] - (x.published ? t : 0);
  const float slope = x.slopes ? x.slopes[h * x.G + g] : 0.f;
  const int lim = n + max(i + 1, x.seqs.prefix[s]);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int kb = k0; kb < min(k1, lim); kb += 32) {
    const int j = kb + lane;
    float w = 0.f;
    if (j < lim && j < k1) {
      const int apart = abs(tot + i - x.pos[slab * x.cap + j]);
      if (x.window == 0 || apart < x.window) {
        float dot = 0.f;
        for (int c = 0; c < 128; ++c)
          dot = fmaf(__bfloat162float(q[c]), ext_row_value<__nv_bfloat16, KV8>(x.K, (slab * x.cap + j) * 128 + c, 1.f), dot);
        w = fast_exp2(ext_logit_exact(x, dot, slope, apart) - m);
      }
    }
    for (int kk = 0; kk < 32; ++kk) {
      const float wk = __shfl_sync(0xffffffffu, w, kk);
      if (wk == 0.f) continue;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        acc[u] = fmaf(wk, ext_row_value<__nv_bfloat16, KV8>(x.V, (slab * x.cap + kb + kk) * 128 + 4 * lane + u, 1.f), acc[u]);
    }
  }
  return make_float4(acc[0], acc[1], acc[2], acc[3]);
}

// The end of an item, by the softmax warps: its output (or its part's) from tensor memory.  A function of its own:
// it runs once per item, and inlined its registers would cost the tile loop spills.
template <bool KV8>
__device__ __noinline__ void xt_epilogue(const ExtendTcParams& p, const XtCursor& c, float m, float l, uint32_t tO, uint32_t bar12,
                                         volatile int* s_abort, uint8_t* s_out) {
  const ExtendParams& x = p.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
  const uint32_t g_inv = 65536u / (uint32_t)x.G + 1u;
  uint8_t* stage = s_out + warp * (32 * 128);
  const int r = tid;

  // The row of O, normalised and rounded: half a row at a time through the warp's staging tile, so that the
  // global stores are whole 128-byte lines (prefill_attn.cuh).
  auto write_half = [&](const XtCursor& c, int c0, const uint32_t (&o)[2][32], float factor) {
    const uint64_t f2 = tc5::f2_pack(factor, factor);
#pragma unroll
    for (int hh = 0; hh < 2; ++hh) {
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        uint32_t w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float y0, y1;
          tc5::f2_unpack(tc5::f2_mul(tc5::f2_pack(__uint_as_float(o[hh][e + 2 * u]), __uint_as_float(o[hh][e + 2 * u + 1])), f2), y0, y1);
          w[u] = pack_bf16x2(y0, y1);
        }
        const int chunk = 4 * hh + (e >> 3);
        *reinterpret_cast<uint4*>(stage + lane * 128 + ((chunk ^ (lane & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    __syncwarp();
    __nv_bfloat16* obase = static_cast<__nv_bfloat16*>(x.out) +
                           (((size_t)c.layer * x.total + x.seqs.tok0[c.s] + c.i0) * x.Hq + c.h * x.G) * 128 + c0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int row = 4 * i + (lane >> 3), chunk = lane & 7;
      const uint4 w = *reinterpret_cast<const uint4*>(stage + row * 128 + ((chunk ^ (row & 7)) << 4));
      const int rr = warp * 32 + row;
      const int ti = (int)((uint32_t)rr * g_inv >> 16);
      if (rr < c.rows && !*s_abort) *reinterpret_cast<uint4*>(obase + ((size_t)ti * x.Hq + (rr - ti * x.G)) * 128 + chunk * 8) = w;
    }
    __syncwarp();
  };
  // Half a row of the unnormalised O from tensor memory; elements that are not finite are computed again.
  auto read_half = [&](const XtCursor& c, int c0, uint32_t (&o)[2][32], float m) {
    tc5::tmem_ld32(tO + lane_base + (uint32_t)c0, o[0]);
    tc5::tmem_ld32(tO + lane_base + (uint32_t)c0 + 32u, o[1]);
    tc5::tmem_wait_ld();
    float probe = 0.f;  // 0 * finite = 0
#pragma unroll
    for (int e = 0; e < 32; ++e) probe = fmaf(__uint_as_float(o[0][e]), 0.f, fmaf(__uint_as_float(o[1][e]), 0.f, probe));
    unsigned again = __ballot_sync(0xffffffffu, !(probe == 0.f) && r < c.rows);
    while (again) {
      const int who = __ffs(again) - 1;
      again &= again - 1;
      const int rr = warp * 32 + who, ti = (int)((uint32_t)rr * g_inv >> 16);
      const float mm = __shfl_sync(0xffffffffu, m, who);
      const float4 y = xt_row_again<KV8>(p, c.s, c.layer, c.h, c.n, c.i0 + ti, rr - ti * x.G, c.kt0 * kPfKeys, (c.kt0 + c.nkt) * kPfKeys, mm);
      __syncwarp();
      reinterpret_cast<float4*>(stage)[lane] = y;
      __syncwarp();
      if (lane == who) {
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          if (!(__uint_as_float(o[0][e]) * 0.f == 0.f)) o[0][e] = reinterpret_cast<const uint32_t*>(stage)[c0 + e];
          if (!(__uint_as_float(o[1][e]) * 0.f == 0.f)) o[1][e] = reinterpret_cast<const uint32_t*>(stage)[c0 + 32 + e];
        }
      }
      __syncwarp();
    }
  };
  const float out_scale = KV8 ? x.v_scale : 1.f;

  mbar_wait(bar12, (uint32_t)(c.ord & 1), s_abort, x.err, kPfSpinLimit);
  tc5::fence_after_sync();
  const bool live = warp * 32 < c.rows;
  uint32_t o[2][32];
  if (c.n_split == 1) {
    if (!live) return;
    const float f = out_scale / l;
#pragma unroll 1
    for (int c0 = 0; c0 < 128; c0 += 64) {
      read_half(c, c0, o, m);
      write_half(c, c0, o, f);
    }
    if (x.lse && r < c.rows) x.lse[ext_lse_index(x, c.layer, c.h, x.seqs.tok0[c.s] + c.i0) + r] = m + __log2f(l);
    return;
  }
  // one of several parts: [32 pieces of four columns][part_rows] float4, then [part_rows] (m, l)
  const size_t piece = (size_t)p.part_rows;
  auto part_of = [&](int split) { return p.part + ((size_t)(c.u0 + split) * p.lh + c.lh) * (piece * kXtPartFloats); };
  if (live) {
    float* mine = part_of(c.split);
#pragma unroll 1
    for (int c0 = 0; c0 < 128; c0 += 64) {
      read_half(c, c0, o, m);
      if (r < c.rows && !*s_abort) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int e = 0; e < 32; e += 4)
            __stcg(reinterpret_cast<float4*>(mine) + (size_t)(c0 / 4 + 8 * hh + e / 4) * piece + r,
                   make_float4(__uint_as_float(o[hh][e]), __uint_as_float(o[hh][e + 1]), __uint_as_float(o[hh][e + 2]), __uint_as_float(o[hh][e + 3])));
      }
    }
    if (r < c.rows && !*s_abort) __stcg(reinterpret_cast<float2*>(mine + 128 * piece) + r, make_float2(m, l));
  }
  __threadfence();
  asm volatile("bar.sync 1, 128;" ::: "memory");
  int* s_last = reinterpret_cast<int*>(s_out);  // (the first warp's staging tile is free here)
  if (tid == 0) *s_last = atomicAdd(x.counters + (size_t)c.u0 * p.lh + c.lh, 1u) == (unsigned)(c.n_split - 1);
  asm volatile("bar.sync 1, 128;" ::: "memory");
  const bool last = *s_last != 0;
  asm volatile("bar.sync 1, 128;" ::: "memory");
  if (!last || !live) return;
  __threadfence();
  const int rr = min(r, c.rows - 1);  // (lanes without a row follow along)
  float M = -CUDART_INF_F;
  for (int k = 0; k < c.n_split; ++k) M = fmaxf(M, __ldcg(reinterpret_cast<const float2*>(part_of(k) + 128 * piece) + rr).x);
  const float M0 = M == -CUDART_INF_F ? 0.f : M;
  float Lsum = 0.f;
  for (int k = 0; k < c.n_split; ++k) {
    const float2 ml = __ldcg(reinterpret_cast<const float2*>(part_of(k) + 128 * piece) + rr);
    Lsum += ml.y * fast_exp2(ml.x - M0);
  }
  const float f = out_scale / Lsum;
#pragma unroll 1
  for (int c0 = 0; c0 < 128; c0 += 64) {
#pragma unroll
    for (int e = 0; e < 32; ++e) o[0][e] = o[1][e] = 0u;
#pragma unroll 1
    for (int k = 0; k < c.n_split; ++k) {
      const float* src = part_of(k);
      const float wk = fast_exp2(__ldcg(reinterpret_cast<const float2*>(src + 128 * piece) + rr).x - M0);
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int e = 0; e < 32; e += 4) {
          const float4 y = __ldcg(reinterpret_cast<const float4*>(src) + (size_t)(c0 / 4 + 8 * hh + e / 4) * piece + rr);
          o[hh][e] = __float_as_uint(fmaf(wk, y.x, __uint_as_float(o[hh][e])));
          o[hh][e + 1] = __float_as_uint(fmaf(wk, y.y, __uint_as_float(o[hh][e + 1])));
          o[hh][e + 2] = __float_as_uint(fmaf(wk, y.z, __uint_as_float(o[hh][e + 2])));
          o[hh][e + 3] = __float_as_uint(fmaf(wk, y.w, __uint_as_float(o[hh][e + 3])));
        }
    }
    write_half(c, c0, o, f);
  }
  if (x.lse && r < c.rows) x.lse[ext_lse_index(x, c.layer, c.h, x.seqs.tok0[c.s] + c.i0) + r] = M + __log2f(Lsum);
}

template <bool KV8, bool MODS>
__global__ void __launch_bounds__(kXtThreads, 2)
extend_tc_kernel(const __grid_constant__ ExtendTcParams p, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV) {
  extern __shared__ __align__(1024) uint8_t pf_smem[];
  uint8_t* sm = pf_smem;
  const uint32_t sQ = smem_u32(sm);                       // [2 halves of head_dim][128 rows][128 B]
  const uint32_t sK = sQ + kPfQBytes;                     // [2 stages][2 halves][64 rows][128 B]
  const uint32_t sV = sK + 2 * kPfKvBytes;                // the same
  uint8_t* s_out = sm + kPfQBytes + 4 * kPfKvBytes;       // [4 softmax warps][32 rows][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_out + kPfOutStageBytes);
  // barriers: 0 Q, 1-2 K stages filled, 3-4 V stages filled, 5-6 S buffers complete, 7 O += P V complete, 8-9 P written
  // (per S buffer), 10-11 V stages read, 12 the item's last O += P V complete, 13-14 drain (see prefill_attn.cuh)
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 15);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_n = reinterpret_cast<int*>(s_out + kPfOutStageBytes + 128);  // rows held by each sequence, -1: the chunk has no room
  const ExtendParams& x = p.x;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int n_items = (p.n_work - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;
  if (tid == 0) {
    for (int i = 0; i < 15; ++i) mbar_init(bar(i), (i == 8 || i == 9) ? kXtRows : 1);
    *s_abort = 0;
    if ((smem_u32(sm) & 1023u) != 0u) {
      atomicOr(x.err, kErrStreamBounds);
      *s_abort = 1;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 5) {
    tc5::tmem_alloc(smem_u32(s_tmem), kPfTmemCols);
    tc5::tmem_relinquish();
  }
  // The storing kernel may still be running; everything below waits until it has completed.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  for (int s = tid; s < x.seqs.n; s += kXtThreads) {
    const ExtSeq e = ext_seq(x, s);
    s_n[s] = e.ok ? e.n : -1;
  }
  tc5::fence_before_sync();
  __syncthreads();
  tc5::fence_after_sync();
  const uint32_t tmem = *s_tmem;
  const uint32_t tS0 = tmem, tO = tmem + 128;  // S buffer b at column 64 b
  XtCursor first;
  first.ord = 0;
  xt_seek(first, 0, n_items, p, s_n);
  auto slab_of = [&](const XtCursor& c) { return ((x.layer0 + c.layer) * x.Nb + x.seqs.b0 + c.s) * x.Hkv + c.h; };
  const uint32_t q_bytes = 256u * (uint32_t)(x.G * p.tokens_per_tile);
  auto load_q = [&](const XtCursor& c) {
    const int tok = c.layer * x.total + x.seqs.tok0[c.s] + c.i0;
    mbar_arrive_expect_tx(bar(0), q_bytes);
    pf_tma_load(sQ, &tmQ, 0, c.h * x.G, tok, bar(0));
    pf_tma_load(sQ + kPfQBytes / 2, &tmQ, 64, c.h * x.G, tok, bar(0));
  };
  auto load_tile = [&](const CUtensorMap* tm, uint32_t base, int bar_i, const XtCursor& c, int g) {
    const uint32_t dst = base + (uint32_t)(g & 1) * kPfKvBytes, bb = bar(bar_i + (g & 1));
    const int row = (c.kt0 + c.j) * kPfKeys, slab = slab_of(c);
    mbar_arrive_expect_tx(bb, kPfKvBytes);
    pf_tma_load(dst, tm, 0, row, slab, bb);
    pf_tma_load(dst + kPfKvBytes / 2, tm, 64, row, slab, bb);
  };
  // 8-bit rows: the loading warps fill a stage themselves
  XtCodes codes;
  auto fetch_codes = [&](const void* base, const XtCursor& c) {
    const int t = x.seqs.tok0[c.s + 1] - x.seqs.tok0[c.s];
    xt_load_codes(codes, static_cast<const uint8_t*>(base) + (size_t)slab_of(c) * x.cap * 128, (c.kt0 + c.j) * kPfKeys, c.n + t, lane);
  };
  auto fill_stage = [&](uint32_t off, int bar_i, int g) {
    xt_store_codes(codes, sm + off + (uint32_t)(g & 1) * kPfKvBytes, kPfKvBytes / 2, lane);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(bar_i + (g & 1)));
    __syncwarp();
  };

  if (warp == 4) {
    // ================= the warp that loads Q and K =================
    if (lane == 0 && *reinterpret_cast<volatile int*>(p.stop) != 0) *s_abort = 1;
    __syncwarp();
    if (first.it < n_items && !*s_abort) {
      if (tc5::elect_one()) load_q(first);
      __syncwarp();
      XtCursor cur = first, cK = first;
      if constexpr (KV8) fetch_codes(x.K, cK);
      for (int g = 0; g < 2 && cK.it < n_items; ++g) {
        if constexpr (KV8) {
          fill_stage(kPfQBytes, 1, g);
          xt_advance(cK, n_items, p, s_n);
          if (cK.it < n_items) fetch_codes(x.K, cK);
        } else {
          if (tc5::elect_one()) load_tile(&tmK, sK, 1, cK, g);
          __syncwarp();
          xt_advance(cK, n_items, p, s_n);
        }
      }
      XtCursor nq = first;  // the item after the current one
      ++nq.ord;
      xt_seek(nq, first.it + 1, n_items, p, s_n);
      for (int g = 0; cur.it < n_items && !*s_abort; ++g) {
        const bool next_q = cur.j == cur.nkt - 1 && nq.it < n_items;
        if (cur.j == 0 && nq.it < n_items && tc5::elect_one()) {
          const int tok = nq.layer * x.total + x.seqs.tok0[nq.s] + nq.i0;
          pf_tma_prefetch(&tmQ, 0, nq.h * x.G, tok);
          pf_tma_prefetch(&tmQ, 64, nq.h * x.G, tok);
        }
        if (cK.it < n_items || next_q) {
          mbar_wait(bar(5 + (g & 1)), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);
          __syncwarp();
          if (*s_abort) break;
          if (next_q && tc5::elect_one()) load_q(nq);
          __syncwarp();
          if (cK.it < n_items) {  // tile g + 2: the stage S_g read
            if constexpr (KV8) {
              fill_stage(kPfQBytes, 1, g);
              xt_advance(cK, n_items, p, s_n);
              if (cK.it < n_items) fetch_codes(x.K, cK);
            } else {
              if (tc5::elect_one()) load_tile(&tmK, sK, 1, cK, g);
              __syncwarp();
              xt_advance(cK, n_items, p, s_n);
            }
          }
        }
        if (cur.j == cur.nkt - 1) {
          cur = nq;
          if (nq.it < n_items) {
            ++nq.ord;
            xt_seek(nq, nq.it + 1, n_items, p, s_n);
          }
        } else {
          ++cur.j;
        }
      }
    }
    if (*s_abort && lane == 0) {
      // Something gave up: a bounded time for the loads this warp started (see prefill_attn.cuh).
      atomicOr(p.stop, 1);
      for (int i = 0; i < (KV8 ? 1 : 3); ++i)
        for (uint32_t ph = 0; ph < 2; ++ph)
          for (uint32_t w = 0; w < (1u << 16); ++w)
            if (mbar_try_wait(bar(i), ph)) break;
    }
  } else if (warp == 7) {
    // ================= the warp that loads V =================
    XtCursor cV = first;
    if constexpr (KV8) {
      if (cV.it < n_items) fetch_codes(x.V, cV);
    }
    for (int g = 0; cV.it < n_items && !*s_abort; ++g) {
      // V of tile g after O += P V of tile g - 2 has completed (the stage it read)
      if (g >= 2) mbar_wait(bar(10 + (g & 1)), (uint32_t)(((g - 2) >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      __syncwarp();
      if (*s_abort) break;
      if constexpr (KV8) {
        fill_stage(kPfQBytes + 2 * kPfKvBytes, 3, g);
        xt_advance(cV, n_items, p, s_n);
        if (cV.it < n_items) fetch_codes(x.V, cV);
      } else {
        if (tc5::elect_one()) load_tile(&tmV, sV, 3, cV, g);
        __syncwarp();
        xt_advance(cV, n_items, p, s_n);
      }
    }
    if (!KV8 && *s_abort && lane == 0) {
      atomicOr(p.stop, 1);
      for (int i = 3; i < 5; ++i)
        for (uint32_t ph = 0; ph < 2; ++ph)
          for (uint32_t w = 0; w < (1u << 16); ++w)
            if (mbar_try_wait(bar(i), ph)) break;
    }
  } else if (warp == 5) {
    // ================= the warp that issues O += P V =================
    constexpr uint32_t idesc_o = KV8 ? tc5::idesc_f16_f32(kXtRows, 128, 0, 1) : tc5::idesc_bf16_f32(kXtRows, 128, 0, 1);
    const uint64_t dV = tc5::smem_desc_sw128(sV, kPfKvBytes / 2, 1024);
    XtCursor cur = first;
    for (int g = 0; cur.it < n_items && !*s_abort; ++g) {
      const int st = g & 1;
      mbar_wait(bar(3 + st), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      mbar_wait(bar(8 + st), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      __syncwarp();
      tc5::fence_after_sync();
      if (*s_abort) break;
      const uint64_t dVg = dV + (uint64_t)((uint32_t)st * (kPfKvBytes >> 4));
      if (tc5::elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          tc5::mma_bf16_ts(tO, tS0 + 64u * (uint32_t)st + 8u * (uint32_t)kk, dVg + (uint64_t)(kk * 128), idesc_o,
                           (cur.j > 0 || kk > 0) ? 1u : 0u);
        tc5::mma_commit(bar(7));
        tc5::mma_commit(bar(10 + st));
        if (cur.j == cur.nkt - 1) tc5::mma_commit(bar(12));
      }
      __syncwarp();
      xt_advance(cur, n_items, p, s_n);
    }
    if (*s_abort && tc5::elect_one()) {
      atomicOr(p.stop, 1);
      tc5::mma_commit(bar(13));
      for (uint32_t w = 0; w < kPfSpinLimit; ++w)
        if (mbar_try_wait(bar(13), 0u)) break;
    }
  } else if (warp == 6) {
    // ================= the warp that issues S = Q K^T =================
    constexpr uint32_t idesc_s = KV8 ? tc5::idesc_f16_f32(kXtRows, kPfKeys, 0, 0) : tc5::idesc_bf16_f32(kXtRows, kPfKeys, 0, 0);
    const uint64_t dQ = tc5::smem_desc_sw128(sQ, 16, 1024);
    const uint64_t dK = tc5::smem_desc_sw128(sK, 16, 1024);
    XtCursor cur = first;
    for (int g = 0; cur.it < n_items && !*s_abort; ++g) {
      const int st = g & 1;
      mbar_wait(bar(1 + st), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      if (g >= 2) mbar_wait(bar(10 + st), (uint32_t)(((g - 2) >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      if (cur.j == 0) mbar_wait(bar(0), (uint32_t)(cur.ord & 1), s_abort, x.err, kPfSpinLimit);
      __syncwarp();
      tc5::fence_after_sync();
      if (!*s_abort) {
        const uint64_t dKg = dK + (uint64_t)((uint32_t)st * (kPfKvBytes >> 4));
        if (tc5::elect_one()) {
#pragma unroll
          for (int kk = 0; kk < 8; ++kk)
            tc5::mma_bf16_ss(tS0 + 64u * (uint32_t)st, dQ + (uint64_t)((kk >> 2) * (kPfQBytes >> 5) + (kk & 3) * 2),
                             dKg + (uint64_t)((kk >> 2) * (kPfKvBytes >> 5) + (kk & 3) * 2), idesc_s, kk > 0);
          tc5::mma_commit(bar(5 + st));
        }
        __syncwarp();
      }
      xt_advance(cur, n_items, p, s_n);
    }
    if (*s_abort && tc5::elect_one()) {
      atomicOr(p.stop, 1);
      tc5::mma_commit(bar(14));
      for (uint32_t w = 0; w < kPfSpinLimit; ++w)
        if (mbar_try_wait(bar(14), 0u)) break;
    }
  } else {
    // ================= softmax warps: thread = query row = tensor-memory lane =================
    const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
    const uint32_t g_inv = 65536u / (uint32_t)x.G + 1u;  // r / G == r * g_inv >> 16 for r < 128
    uint8_t* stage = s_out + warp * (32 * 128);
    const int r = tid;                                    // query row within the tile
    const int ri = (int)((uint32_t)r * g_inv >> 16), rg = r - ri * x.G;

    bool ep_on = false;  // an item whose epilogue is still to run, and what it needs
    XtCursor ep_c = first;
    float ep_m = 0.f, ep_l = 0.f;
    XtCursor cur = first;
    int g = 0;  // flat tile index: S buffer g & 1
    while (cur.it < n_items) {
      const bool live = warp * 32 < cur.rows;
      const int prefix = x.seqs.prefix[cur.s];
      const int row_c = min(r, cur.rows - 1);  // (a lane without a query repeats the last row's visibility)
      const int ti = cur.i0 + (int)((uint32_t)row_c * g_inv >> 16);
      const int lim = cur.n + max(ti + 1, prefix);  // rows [0, lim) are visible
      const int lim_min = __shfl_sync(0xffffffffu, lim, 0), lim_max = __shfl_sync(0xffffffffu, lim, 31);
      // MODS: positions relative to the chunk's first token, two per lane, one tile ahead
      const int* pos_row = nullptr;
      int tot = 0, pos_a = 0, pos_b = 0;
      float slope = 0.f;
      if constexpr (MODS) {
        const int b = x.seqs.b0 + cur.s, t = x.seqs.tok0[cur.s + 1] - x.seqs.tok0[cur.s];
        tot = x.tot[b] - (x.published ? t : 0);
        pos_row = x.pos + (size_t)slab_of(cur) * x.cap;
        if (x.slopes) slope = x.slopes[cur.h * x.G + rg] * 1.4426950408889634f;
        pos_a = pos_row[min(cur.kt0 * kPfKeys + lane, x.cap - 1)] - tot;
        pos_b = pos_row[min(cur.kt0 * kPfKeys + 32 + lane, x.cap - 1)] - tot;
      }
      float m = -CUDART_INF_F, l = 0.f;
      for (int j = 0; j < cur.nkt; ++j, ++g) {
        const int key0 = (cur.kt0 + j) * kPfKeys;
        uint32_t s_lo[32], s_hi[32];
        uint32_t pk[32];  // the row's 64 weights as 16-bit pairs
        bool move = false;
        float alpha = 1.f;
        mbar_wait(bar(5 + (g & 1)), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);  // S of this tile is complete
        tc5::fence_after_sync();
        if (live) {
          tc5::tmem_ld32(tS0 + lane_base + 64u * (uint32_t)(g & 1), s_lo);
          tc5::tmem_ld32(tS0 + lane_base + 64u * (uint32_t)(g & 1) + 32u, s_hi);
          bool border = false;
          const int* ipos = nullptr;
          if constexpr (MODS) {
            ipos = reinterpret_cast<const int*>(stage);
            float* fpos = reinterpret_cast<float*>(stage) + 64;
            __syncwarp();
            reinterpret_cast<int*>(stage)[lane] = pos_a;
            reinterpret_cast<int*>(stage)[32 + lane] = pos_b;
            fpos[lane] = (float)pos_a;
            fpos[32 + lane] = (float)pos_b;
            if (x.window > 0) {
              // the first and last position of the tile against the warp's first and last token
              const int p0 = __shfl_sync(0xffffffffu, pos_a, 0), p1 = __shfl_sync(0xffffffffu, pos_b, 31);
              const int ta = __shfl_sync(0xffffffffu, ti, 0), tb = __shfl_sync(0xffffffffu, ti, 31);
              border = key0 + kPfKeys > cur.n || (long long)tb - p0 >= x.window || (long long)p1 - ta >= x.window;
            }
            if (j + 1 < cur.nkt) {
              pos_a = pos_row[min(key0 + kPfKeys + lane, x.cap - 1)] - tot;
              pos_b = pos_row[min(key0 + kPfKeys + 32 + lane, x.cap - 1)] - tot;
            }
            __syncwarp();
          }
          tc5::tmem_wait_ld();
          float scale_log2 = p.scale_log2;
          if constexpr (MODS) {
            const float* fpos = reinterpret_cast<const float*>(stage) + 64;
            const float fi = (float)ti;
            auto modify = [&](uint32_t (&sv)[32], int hb) {
              if (x.cap_logit > 0.f) {  // c tanh(y) = c - 2 c / (1 + e^(2 y))
#pragma unroll
                for (int c = 0; c < 32; ++c)
                  sv[c] = __float_as_uint(fmaf(-2.f * p.cap_log2, rcp_approx(1.f + fast_exp2(__uint_as_float(sv[c]) * p.cap_arg)), p.cap_log2));
              } else {
#pragma unroll
                for (int c = 0; c < 32; ++c) sv[c] = __float_as_uint(__uint_as_float(sv[c]) * p.scale_log2);
              }
              if (x.slopes) {
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                  const float4 f = *reinterpret_cast<const float4*>(fpos + hb + c);
                  sv[c] = __float_as_uint(fmaf(-slope, fabsf(fi - f.x), __uint_as_float(sv[c])));
                  sv[c + 1] = __float_as_uint(fmaf(-slope, fabsf(fi - f.y), __uint_as_float(sv[c + 1])));
                  sv[c + 2] = __float_as_uint(fmaf(-slope, fabsf(fi - f.z), __uint_as_float(sv[c + 2])));
                  sv[c + 3] = __float_as_uint(fmaf(-slope, fabsf(fi - f.w), __uint_as_float(sv[c + 3])));
                }
              }
              if (border) {
#pragma unroll
                for (int c = 0; c < 32; ++c)
                  if (abs(ti - ipos[hb + c]) >= x.window) sv[c] = 0xff800000u;
              }
            };
            modify(s_lo, 0);
            modify(s_hi, 32);
            scale_log2 = 1.f;
          }
          // The mask, per warp and half tile: a half is fully visible, hidden, or compared column by column.
          const int cv = lim - key0, cv_min = lim_min - key0, cv_max = lim_max - key0;
          const bool lo_live = cv_max > 0, hi_live = cv_max > 32;
          if (cv_min < 32) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (c >= cv) s_lo[c] = 0xff800000u;  // -inf
          }
          if (hi_live && cv_min < 64) {
#pragma unroll
            for (int c = 0; c < 32; ++c)
              if (c + 32 >= cv) s_hi[c] = 0xff800000u;
          }
          auto max_half = [](const uint32_t (&sv)[32]) {  // four chains of three-input maxima
            float mx4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
            for (int c = 0; c < 32; c += 8) {
#pragma unroll
              for (int u = 0; u < 4; ++u) mx4[u] = tc5::f_max3(mx4[u], __uint_as_float(sv[c + u]), __uint_as_float(sv[c + 4 + u]));
            }
            return tc5::f_max3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]);
          };
          float mxr = -CUDART_INF_F;
          if (lo_live) mxr = max_half(s_lo);
          if (hi_live) mxr = fmaxf(mxr, max_half(s_hi));
          const float mx = mxr * scale_log2;
          // the reference maximum moves only when it is exceeded by more than 2^8 (see prefill_attn.cuh); a row that
          // has seen nothing yet keeps -inf and weighs with exp2(-inf - 0) = 0
          move = mx > m + 8.0f && r < cur.rows;
          const float m_new = move ? mx : m;
          alpha = move ? fast_exp2(m - m_new) : 1.0f;
          const float neg_m = m_new == -CUDART_INF_F ? 0.f : -m_new;
          const uint64_t scale2 = tc5::f2_pack(scale_log2, scale_log2), negm2 = tc5::f2_pack(neg_m, neg_m);
          auto exp_half = [scale2, negm2](const uint32_t (&sv)[32], uint32_t* out) {
            uint64_t sum2[4] = {0ull, 0ull, 0ull, 0ull};  // four chains of (even, odd) column sums
#pragma unroll
            for (int c = 0; c < 16; ++c) {
              float x0, x1;
              tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[2 * c]), __uint_as_float(sv[2 * c + 1])), scale2, negm2), x0, x1);
              const float a0 = fast_exp2(x0), a1 = fast_exp2(x1);
              sum2[c & 3] = tc5::f2_add(sum2[c & 3], tc5::f2_pack(a0, a1));
              out[c] = KV8 ? pack_f16x2(a0, a1) : pack_bf16x2(a0, a1);
            }
            float e, o;
            tc5::f2_unpack(tc5::f2_add(tc5::f2_add(sum2[0], sum2[1]), tc5::f2_add(sum2[2], sum2[3])), e, o);
            return e + o;
          };
          float sum = 0.f;
          if (lo_live) {
            sum = exp_half(s_lo, pk);
          } else {
#pragma unroll
            for (int c = 0; c < 16; ++c) pk[c] = 0u;
          }
          if (hi_live) {
            sum += exp_half(s_hi, pk + 16);
          } else {
#pragma unroll
            for (int c = 0; c < 16; ++c) pk[16 + c] = 0u;
          }
          l = l * alpha + sum;
          m = m_new;
          if (j > 0 && __any_sync(0xffffffffu, move)) {
            // O += P V of the tile before must be complete before O is rescaled (see prefill_attn.cuh)
            mbar_wait(bar(7), (uint32_t)((g - 1) & 1), s_abort, x.err, kPfSpinLimit);
            tc5::fence_after_sync();
#pragma unroll
            for (int c0 = 0; c0 < 128; c0 += 32) {
              uint32_t o[32];
              tc5::tmem_ld32(tO + lane_base + (uint32_t)c0, o);
              tc5::tmem_wait_ld();
#pragma unroll
              for (int c = 0; c < 32; ++c) o[c] = __float_as_uint(__uint_as_float(o[c]) * alpha);
              tc5::tmem_st32(tO + lane_base + (uint32_t)c0, o);
            }
          }
        }
        // The epilogue of the item before runs here, while its last O += P V completes; the first O = P V of
        // this item cannot be issued before the P stored below.
        if (ep_on) {
          xt_epilogue<KV8>(p, ep_c, ep_m, ep_l, tO, bar(12), s_abort, s_out);
          ep_on = false;
        }
        if (live) {
          tc5::tmem_st32(tS0 + lane_base + 64u * (uint32_t)(g & 1), pk);
          tc5::tmem_wait_st();
        }
        tc5::fence_before_sync();
        mbar_arrive(bar(8 + (g & 1)));
      }
      ep_on = true;
      ep_c = cur;
      ep_m = m;
      ep_l = l;
      ++cur.ord;
      xt_seek(cur, cur.it + 1, n_items, p, s_n);
    }
    if (ep_on) xt_epilogue<KV8>(p, ep_c, ep_m, ep_l, tO, bar(12), s_abort, s_out);
  }
  tc5::fence_before_sync();
  __syncthreads();
  if (warp == 5) tc5::tmem_dealloc(tmem, kPfTmemCols);
}

// extend_mass_tc_kernel: mass_j = sum over the chunk's tokens i and the group's heads of exp2(x_ij - lse_i).
// The products are taken the other way round -- M = 128 keys, N = 64 query rows -- so that thread = key = tensor-
// memory lane: the sum over the queries stays in one register, needs no exchange between lanes and no atomics, and
// exactly one thread writes a row.  A work item = 128 rows of one slab against all query rows that see any of them;
// persistent CTAs, two per SM.  K tiles (two stages, the next item's asked for when the item begins) and Q tiles (two
// stages of 64 rows) by TMA, S in two buffers of 64 columns.  Bound by the exponentials like the attention itself.
constexpr int kXmKeys = 128;
constexpr int kXmRows = 64;                       // query rows per step
constexpr int kXmKBytes = kXmKeys * 256;
constexpr int kXmQBytes = kXmRows * 256;
constexpr int kXmWarpFloats = 128;                // per compute warp: 64 negated log-sum-exps, 64 slopes
constexpr int kXmSmemBytes = 2 * kXmKBytes + 2 * kXmQBytes + 128 + 4 * kXmWarpFloats * 4 + kXmRows * 4 + kExtSeqs * 4 + (kExtSeqs + 1) * 4 + 12;
constexpr uint32_t kXmTmemCols = 128;

struct XmCursor {
  int it, ord;        // position in this CTA's list; items with steps before it
  int j, lo, n_step;  // step within the item, first query tile, query tiles
  int s, layer, h, n, t, k0;
};

struct XmShared {
  const int* n;      // rows held by each sequence
  const int* item0;  // first (sequence, key tile) of each sequence
  int n_work;
};

__device__ __forceinline__ void xm_seek(XmCursor& c, int it, int n_items, const ExtendTcParams& p, const XmShared& sh, bool skip_empty) {
  c.j = 0;
  const int tps = kXmRows / p.x.G;  // tokens per step
  for (; it < n_items; ++it) {
    const int w = (int)blockIdx.x + it * (int)gridDim.x;
    const int u = w / p.lh, lh = w - u * p.lh;
    c.s = ext_find(sh.item0, p.x.seqs.n, u);
    c.n = sh.n[c.s];
    c.t = p.x.seqs.tok0[c.s + 1] - p.x.seqs.tok0[c.s];
    c.k0 = (u - sh.item0[c.s]) * kXmKeys;
    c.layer = lh / p.x.Hkv;
    c.h = lh - c.layer * p.x.Hkv;
    c.lo = c.k0 < c.n + p.x.seqs.prefix[c.s] ? 0 : (c.k0 - c.n) / tps;
    int hi = (c.t + tps - 1) / tps;
    if (p.x.window > 0) {  // a token is at least as many positions behind a row as it is rows behind it
      const long long last = (long long)p.x.window + c.k0 + kXmKeys - 1 - c.n;  // tokens from here on see none of the rows
      hi = last <= 0 ? 0 : (int)min((long long)hi, (last + tps - 1) / tps);
    }
    c.n_step = max(0, hi - c.lo);
    if (c.n_step > 0 || !skip_empty) break;
  }
  c.it = it;
}

template <bool KV8, bool MODS>
__global__ void __launch_bounds__(kXtThreads, 2)
extend_mass_tc_kernel(const __grid_constant__ ExtendTcParams p, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK) {
  extern __shared__ __align__(1024) uint8_t pf_smem[];
  uint8_t* sm = pf_smem;
  const uint32_t sK = smem_u32(sm);             // [2 stages][2 halves of head_dim][128 rows][128 B]
  const uint32_t sQ = sK + 2 * kXmKBytes;       // [2 stages][2 halves][64 rows][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + 2 * kXmKBytes + 2 * kXmQBytes);
  // barriers: 0-1 K stages filled, 2-3 Q stages filled, 4-5 S buffers complete, 6-7 S buffers read, 8-9 K stages read, 10 drain
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 15);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  float* s_warp = reinterpret_cast<float*>(bars + 16);
  float* s_tok = s_warp + 4 * kXmWarpFloats;    // token of a column within its step
  int* s_n = reinterpret_cast<int*>(s_tok + kXmRows);
  int* s_item0 = s_n + kExtSeqs;
  const ExtendParams& x = p.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int tps = kXmRows / x.G;

  if (tid == 0) {
    for (int i = 0; i < 11; ++i) mbar_init(bar(i), i < 2 && KV8 ? 2 : (i == 6 || i == 7) ? kXmKeys : 1);
    *s_abort = 0;
    if ((smem_u32(sm) & 1023u) != 0u) {
      atomicOr(x.err, kErrStreamBounds);
      *s_abort = 1;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 5) {
    tc5::tmem_alloc(smem_u32(s_tmem), kXmTmemCols);
    tc5::tmem_relinquish();
  }
  if (tid < kXmRows) s_tok[tid] = (float)(tid / x.G);
  // Columns of a step that hold no query (64 is not a multiple of G): no load writes their rows of the Q tiles, which
  // are zero from here on, and their log-sum-exp is +inf, so that they weigh nothing.
  {
    const int pad = kXmRows - tps * x.G;
    for (int i = tid; i < 4 * pad * 8; i += kXtThreads) {
      const int chunk = i & 7, r = tps * x.G + (i >> 3) % pad, half_stage = (i >> 3) / pad;
      *reinterpret_cast<uint4*>(sm + 2 * kXmKBytes + half_stage * (kXmQBytes / 2) + r * 128 + chunk * 16) = make_uint4(0u, 0u, 0u, 0u);
    }
    if (pad > 0) asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  // Items from the lengths on the device (a replayed graph may hold longer sequences than its capture): key tiles
  // per sequence, summed up by one warp.
  if (warp == 0) {
    int before = 0;
    for (int s0 = 0; s0 < x.seqs.n; s0 += 32) {
      const int s = s0 + lane;
      int v = 0;
      if (s < x.seqs.n) {
        const ExtSeq e = ext_seq(x, s);
        s_n[s] = e.n;
        v = e.ok && e.t > 0 ? (e.n + e.t + kXmKeys - 1) / kXmKeys : 0;
      }
      int sum = v;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += y;
      }
      if (s < x.seqs.n) s_item0[s] = before + sum - v;
      before += __shfl_sync(0xffffffffu, sum, 31);
    }
    if (lane == 0) s_item0[x.seqs.n] = before;
  }
  tc5::fence_before_sync();
  __syncthreads();
  tc5::fence_after_sync();
  const uint32_t tmem = *s_tmem;
  const XmShared sh{s_n, s_item0, s_item0[x.seqs.n] * p.lh};
  const int n_items = max(0, (sh.n_work - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x);
  auto slab_of = [&](const XmCursor& c) { return ((x.layer0 + c.layer) * x.Nb + x.seqs.b0 + c.s) * x.Hkv + c.h; };
  auto next = [&](XmCursor& c) {  // the step after this one
    if (++c.j == c.n_step) {
      ++c.ord;
      xm_seek(c, c.it + 1, n_items, p, sh, true);
    }
  };

  if (warp == 4) {
    // ================= the warp that loads Q, and K of 16-bit rows =================
    if (lane == 0 && *reinterpret_cast<volatile int*>(p.stop) != 0) *s_abort = 1;
    __syncwarp();
    XmCursor cur, cK;
    cur.ord = 0;
    xm_seek(cur, 0, n_items, p, sh, true);
    cK = cur;
    auto load_k = [&]() {  // the item of cK; its stage is read by the item two before
      if (cK.ord >= 2) mbar_wait(bar(8 + (cK.ord & 1)), (uint32_t)(((cK.ord - 2) >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      __syncwarp();
      if (!*s_abort && tc5::elect_one()) {
        const uint32_t dst = sK + (uint32_t)(cK.ord & 1) * kXmKBytes, bb = bar(cK.ord & 1);
        const int slab = slab_of(cK);
        mbar_arrive_expect_tx(bb, kXmKBytes);
#pragma unroll
        for (int q = 0; q < 4; ++q)  // (boxes of 64 rows x 64 elements, as the attention's; those behind the slab's end come back as zeros)
          pf_tma_load(dst + (q >> 1) * (kXmKBytes / 2) + (q & 1) * (kXmKBytes / 4), &tmK, 64 * (q >> 1), cK.k0 + 64 * (q & 1), slab, bb);
      }
      __syncwarp();
      ++cK.ord;
      xm_seek(cK, cK.it + 1, n_items, p, sh, true);
    };
    if constexpr (!KV8) {
      if (cK.it < n_items && !*s_abort) load_k();
    }
    for (int g = 0; cur.it < n_items && !*s_abort; ++g) {
      if (g >= 2) mbar_wait(bar(4 + (g & 1)), (uint32_t)(((g - 2) >> 1) & 1), s_abort, x.err, kPfSpinLimit);  // S of step g - 2 has read the stage
      __syncwarp();
      if (*s_abort) break;
      if (tc5::elect_one()) {
        const uint32_t dst = sQ + (uint32_t)(g & 1) * kXmQBytes, bb = bar(2 + (g & 1));
        const int tok = cur.layer * x.total + x.seqs.tok0[cur.s] + (cur.lo + cur.j) * tps;
        mbar_arrive_expect_tx(bb, 256u * (uint32_t)(x.G * tps));
        pf_tma_load(dst, &tmQ, 0, cur.h * x.G, tok, bb);
        pf_tma_load(dst + kXmQBytes / 2, &tmQ, 64, cur.h * x.G, tok, bb);
      }
      __syncwarp();
      if constexpr (!KV8) {
        if (cur.j == 0 && cK.it < n_items) load_k();  // the next item's rows
      }
      next(cur);
    }
    if (*s_abort && lane == 0) {
      atomicOr(p.stop, 1);
      for (int i = KV8 ? 2 : 0; i < 4; ++i)
        for (uint32_t ph = 0; ph < 2; ++ph)
          for (uint32_t w = 0; w < (1u << 16); ++w)
            if (mbar_try_wait(bar(i), ph)) break;
    }
  } else if (warp == 5) {
    // ================= the warp that issues S = K Q^T =================
    constexpr uint32_t idesc = KV8 ? tc5::idesc_f16_f32(kXmKeys, kXmRows, 0, 0) : tc5::idesc_bf16_f32(kXmKeys, kXmRows, 0, 0);
    const uint64_t dK = tc5::smem_desc_sw128(sK, 16, 1024);
    const uint64_t dQ = tc5::smem_desc_sw128(sQ, 16, 1024);
    XmCursor cur;
    cur.ord = 0;
    xm_seek(cur, 0, n_items, p, sh, true);
    for (int g = 0; cur.it < n_items && !*s_abort; ++g) {
      const int st = g & 1, ks = cur.ord & 1;
      if (cur.j == 0) mbar_wait(bar(ks), (uint32_t)((cur.ord >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      mbar_wait(bar(2 + st), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      if (g >= 2) mbar_wait(bar(6 + st), (uint32_t)(((g - 2) >> 1) & 1), s_abort, x.err, kPfSpinLimit);
      __syncwarp();
      tc5::fence_after_sync();
      if (*s_abort) break;
      const uint64_t dKg = dK + (uint64_t)((uint32_t)ks * (kXmKBytes >> 4)), dQg = dQ + (uint64_t)((uint32_t)st * (kXmQBytes >> 4));
      if (tc5::elect_one()) {
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          tc5::mma_bf16_ss(tmem + 64u * (uint32_t)st, dKg + (uint64_t)((kk >> 2) * (kXmKBytes >> 5) + (kk & 3) * 2),
                           dQg + (uint64_t)((kk >> 2) * (kXmQBytes >> 5) + (kk & 3) * 2), idesc, kk > 0);
        tc5::mma_commit(bar(4 + st));
        if (cur.j == cur.n_step - 1) tc5::mma_commit(bar(8 + ks));
      }
      __syncwarp();
      next(cur);
    }
    if (*s_abort && tc5::elect_one()) {
      atomicOr(p.stop, 1);
      tc5::mma_commit(bar(10));
      for (uint32_t w = 0; w < kPfSpinLimit; ++w)
        if (mbar_try_wait(bar(10), 0u)) break;
    }
  } else if (warp >= 6) {
    // ================= 8-bit rows: two warps widen the codes of a K tile, 64 rows each =================
    if constexpr (KV8) {
      XmCursor cK;
      cK.ord = 0;
      xm_seek(cK, 0, n_items, p, sh, true);
      XtCodes codes;
      const int sub = 64 * (warp - 6);
      auto fetch = [&]() {
        xt_load_codes(codes, static_cast<const uint8_t*>(x.K) + (size_t)slab_of(cK) * x.cap * 128, cK.k0 + sub, cK.n + cK.t, lane);
      };
      if (cK.it < n_items) fetch();
      while (cK.it < n_items && !*s_abort) {
        if (cK.ord >= 2) mbar_wait(bar(8 + (cK.ord & 1)), (uint32_t)(((cK.ord - 2) >> 1) & 1), s_abort, x.err, kPfSpinLimit);
        __syncwarp();
        if (*s_abort) break;
        xt_store_codes(codes, sm + (size_t)(cK.ord & 1) * kXmKBytes + sub * 128, kXmKBytes / 2, lane);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(cK.ord & 1));
        __syncwarp();
        ++cK.ord;
        xm_seek(cK, cK.it + 1, n_items, p, sh, true);
        if (cK.it < n_items) fetch();
      }
    }
  } else {
    // ================= compute warps: thread = key = tensor-memory lane =================
    const uint32_t lane_base = (uint32_t)(warp * 32) << 16;
    float* s_lse = s_warp + warp * kXmWarpFloats;  // negated
    float* s_slope = s_lse + kXmRows;
    XmCursor cur;
    cur.ord = 0;
    xm_seek(cur, 0, n_items, p, sh, false);
    int g = 0;
    while (cur.it < n_items) {
      const int j = cur.k0 + tid;
      const bool mine = j < cur.n + cur.t;
      const size_t row = (size_t)slab_of(cur) * x.cap + j;
      const int prefix = x.seqs.prefix[cur.s];
      // the tokens that see row j: [i_lo, i_hi)
      int i_lo = j < cur.n + prefix ? 0 : j - cur.n, i_hi = mine ? cur.t : 0;
      float rel = 0.f;
      if constexpr (MODS) {
        const int b = x.seqs.b0 + cur.s;
        const int at = mine ? x.pos[row] - (x.tot[b] - (x.published ? cur.t : 0)) : 0;  // the row's position, the chunk's first token being 0
        rel = (float)at;
        if (x.window > 0) {
          i_lo = max(i_lo, at - x.window + 1);
          i_hi = (int)min((long long)i_hi, max(0ll, (long long)at + x.window));
        }
        __syncwarp();
        s_slope[lane] = x.slopes ? x.slopes[cur.h * x.G + lane % x.G] * 1.4426950408889634f : 0.f;
        s_slope[32 + lane] = x.slopes ? x.slopes[cur.h * x.G + (32 + lane) % x.G] * 1.4426950408889634f : 0.f;
        __syncwarp();
      }
      const float* lse = x.lse + ext_lse_index(x, cur.layer, cur.h, x.seqs.tok0[cur.s]);
      const int all_rows = cur.t * x.G, step_rows = tps * x.G;
      auto ask = [&](int step, int off) {  // a step's log-sum-exp of column lane + off
        const int r = (cur.lo + step) * step_rows + lane + off;
        return lane + off < step_rows && r < all_rows ? -__ldg(lse + r) : -CUDART_INF_F;
      };
      float la = 0.f, lb = 0.f;
      if (cur.n_step > 0) {
        la = ask(0, 0);
        lb = ask(0, 32);
      }
      float total = 0.f;
      for (int st = 0; st < cur.n_step; ++st, ++g) {
        __syncwarp();
        s_lse[lane] = la;
        s_lse[32 + lane] = lb;
        if (st + 1 < cur.n_step) {
          la = ask(st + 1, 0);
          lb = ask(st + 1, 32);
        }
        __syncwarp();
        const int i0 = (cur.lo + st) * tps;
        const int rows = min(step_rows, all_rows - (cur.lo + st) * step_rows);
        const int c_lo = min(64, max(0, (i_lo - i0) * x.G)), c_hi = min(rows, max(0, (min(i_hi, i0 + tps) - i0) * x.G));
        const bool full = __all_sync(0xffffffffu, c_lo == 0 && c_hi == step_rows);
        const float off0 = (float)i0 - rel;
        mbar_wait(bar(4 + (g & 1)), (uint32_t)((g >> 1) & 1), s_abort, x.err, kPfSpinLimit);
        tc5::fence_after_sync();
        uint64_t sum2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
        for (int hb = 0; hb < 64; hb += 32) {
          uint32_t sv[32];
          tc5::tmem_ld32(tmem + lane_base + 64u * (uint32_t)(g & 1) + (uint32_t)hb, sv);
          tc5::tmem_wait_ld();
          if (hb == 32) {  // both halves are in registers: the buffer may be written again
            tc5::fence_before_sync();
            mbar_arrive(bar(6 + (g & 1)));
          }
          float scale = p.scale_log2;
          if constexpr (MODS) {
            if (x.cap_logit > 0.f) {
              scale = 1.f;
#pragma unroll
              for (int c = 0; c < 32; ++c)
                sv[c] = __float_as_uint(fmaf(-2.f * p.cap_log2, rcp_approx(1.f + fast_exp2(__uint_as_float(sv[c]) * p.cap_arg)), p.cap_log2));
            }
            if (x.slopes) {
#pragma unroll
              for (int c = 0; c < 32; ++c)
                sv[c] = __float_as_uint(fmaf(-s_slope[hb + c], fabsf(off0 + s_tok[hb + c]), __uint_as_float(sv[c]) * scale));
              scale = 1.f;
            }
          }
          const uint64_t scale2 = tc5::f2_pack(scale, scale);
          auto add_up = [&](auto masked) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              const float4 nl = *reinterpret_cast<const float4*>(s_lse + hb + c);
              float y[4];
              tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), scale2, tc5::f2_pack(nl.x, nl.y)), y[0], y[1]);
              tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[c + 2]), __uint_as_float(sv[c + 3])), scale2, tc5::f2_pack(nl.z, nl.w)), y[2], y[3]);
              if constexpr (decltype(masked)::value) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                  if (hb + c + u < c_lo || hb + c + u >= c_hi) y[u] = -CUDART_INF_F;  // weight 0, whatever the logit is
              }
              sum2[(c >> 1) & 3] = tc5::f2_add(sum2[(c >> 1) & 3], tc5::f2_pack(fast_exp2(y[0]), fast_exp2(y[1])));
              sum2[((c >> 1) + 1) & 3] = tc5::f2_add(sum2[((c >> 1) + 1) & 3], tc5::f2_pack(fast_exp2(y[2]), fast_exp2(y[3])));
            }
          };
          if (full) add_up(std::false_type{});
          else add_up(std::true_type{});
        }
        float e, o;
        tc5::f2_unpack(tc5::f2_add(tc5::f2_add(sum2[0], sum2[1]), tc5::f2_add(sum2[2], sum2[3])), e, o);
        total += e + o;
      }
      if (mine && !*s_abort) ext_emit_mass(x, row, total);
      if (cur.n_step > 0) ++cur.ord;
      xm_seek(cur, cur.it + 1, n_items, p, sh, false);
    }
  }
  tc5::fence_before_sync();
  __syncthreads();
  if (warp == 5) tc5::tmem_dealloc(tmem, kXmTmemCols);
}

}  // namespace dynts
