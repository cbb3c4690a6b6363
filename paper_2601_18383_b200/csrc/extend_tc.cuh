// Tensor-core kernels of the chunk operators (definitions in extend.cuh) for head_dim 128, bf16 rows or
// 8-bit rows: tcgen05.mma with the accumulators in tensor memory.
//
// extend_tc_kernel.  A tile of 128 query rows packs the group's G heads of floor(128 / G) neighbouring
// tokens, so a row of K and V is read once for all of them whatever the chunk's length.  An item = (tile of
// query rows, KV head, layer, sequence).  All items' key tiles form one list, of which every CTA takes an equal
// contiguous piece: few tokens behind a long cache, many ragged sequences and a whole prompt are cut alike.
// An item that lies across CTAs is computed in parts side by side; each part leaves its normalised output and
// log-sum-exp in the scratch, and extend_join_kernel joins them in the order of the list.  (The last part to finish
// joined them at first: one CTA then read all parts of its items, up to 20 us after the others had ended.)  Where the
// join would cost more than it evens out, the pieces are whole items (the host's plan says which; it has the figures).
// Two CTAs per SM; per 64 keys
//     S  = Q K^T      M 128 x N 64 x K 128     operands from shared memory
//     P  = exp2(S * scale - ref)               softmax warps, thread = query row = tensor-memory lane
//     O += P V        M 128 x N 128 x K 64     P from tensor memory
//
// What bounds a tile is the chain wait - read S - exponentials - write P of a softmax warp (about 1700 cycles when one
// group of four warps did every tile, against 512 for the two products and 512 for the exponentials' unit), so
// two groups of four warps take the tiles in turn and four warps per scheduler hide one another's waits.  Both need
// the same reference of a row's exponents without talking to each other, so it is fixed: the key tiles are
// walked from the newest to the oldest, the first group takes the first tile (and, where a chunk's tokens see
// different parts of it, the next ones until every token sees one whole tile), sets the reference kXtHeadroom
// above the largest logit met there and hands it over.  Weights are bf16 (exponent range of fp32), so the logits
// of the other tiles may lie up to 2^100 above the reference before a sum leaves the range; a row that does is
// computed again by its warp alone, with a running maximum.  No maximum and no rescale in any other tile.
// (From the newest tile on, because a distance bias only lowers the logits of older rows, and a window hides the oldest.)
//
// Warps: 0-3 and 4-7 the two groups, one that issues S, one that issues O, two that load (see XtShape); they meet through
// mbarriers as in the prompt attention (prefill_attn.cuh), the S buffer, stages and phases follow the flat tile index g.  Every warp
// walks the CTA's pieces by the plan the storing kernel wrote (extend.cuh), a word per lane, the next piece's
// prefetched.  Two CTAs of 384 threads leave 80 registers per thread and hardly any L1: code that spills or does
// not stay in the instruction caches cost several times its instructions, so the loops are rolled, the end of a piece
// is a function of its own, and what is rare is called once from its end (spills: 32 bytes in the plain kernel, none with caps
// and biases, 16 and 36 with 8-bit rows).  4096 tokens behind 4096 rows: 433 us a call with changing inputs, 0.95 PFLOP/s; 375 to
// 395 us replayed on one state, 1.04 to 1.10 PFLOP/s, 0.65 to 0.68 of what cuBLAS reaches.  (Cursors in registers and everything
// unrolled: 453 us when this stood at 388.)  The tensor cores and the exponentials' unit are each busy for a little more than
// half of that time, in turns that the chain of a tile does not let overlap further: tiles of 128 keys with one S buffer,
// or P over another CTA's wait, measured 2 to 12 us more.  Short items are bound by their own chain, about 7 us from the
// load of Q to the store of the output, two of them per SM at a time.
//
// Rows of 16 bits arrive by TMA from the slabs.  8-bit rows (KV8) are read as codes and widened into the same swizzled
// tiles: K to f16 (exact; queries are an f16 copy made by the storing kernel) by the two loading warps, a tile ahead in
// registers; V to bf16 (exact; f16 weights would have no room for the fixed reference, so the weights are rounded to 8 bits
// here where a decode step over the same rows keeps 11) by the group that weighs the tile, while it waits for S.  The codes of coming tiles are asked into L2 meanwhile.
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

// 8-bit rows, and the plain row arithmetic: two warps of their own load (12 warps, 80 registers per thread).  With caps, biases
// and windows the row arithmetic needs the registers more: the warps that issue the products load too (10 warps, 96).
// (Loading warps against none: 4096 behind 4096, plain, 374 us against 455 us; ragged prompts with a bias 109 against 108 us, 1500
// capped tokens 136 against 133 us.)
template <bool KV8, bool MODS>
struct XtShape {
  static constexpr bool kLoaders = KV8 || !MODS;
  static constexpr int kThreads = kLoaders ? 384 : 320;
};
constexpr int kXtRows = 128;
constexpr int kXtMaxCtas = 380;      // CTAs of a launch (two per SM)
constexpr int kXtPartFloats = 129;   // per query row of a part: 128 outputs, log-sum-exp
constexpr float kXtHeadroom = 40.f;  // the reference lies so far (base-2 units) above the first tiles' maximum
constexpr float kXtSumMax = 1.2676506e30f;  // 2^100: a row whose sum of weights exceeds it is computed again
constexpr int kXtStageBytes = 2048;  // per softmax warp
constexpr int kXtSmemBytes = kPfQBytes + 4 * kPfKvBytes + 8 * kXtStageBytes + 128 + 16;

struct ExtendTcParams {
  ExtendParams x;
  ExtendPlan plan;
  int part_rows;        // query rows a part's scratch has room for
  float* part;          // [2 per CTA]: [32][part_rows] float4, [part_rows] float
  int* stop;
  unsigned int wait_limit;  // polls of a bounded wait, at least 2048
  int mass_parts;       // parts the query rows of a mass item are cut into, while there are at most mass_items items
  int mass_items;
  float* mass_part;     // [mass_items][mass_parts][256]
  unsigned int* mass_counters;  // [mass_items], cleared by the storing kernel
  float out_scale;      // v_scale for 8-bit rows
  float scale_log2;     // log2(e) * scale
  float cap_log2;       // c * log2(e)
  float cap_arg;        // 2 log2(e) * scale / c
  float cap_y;          // scale / c
};

__device__ __forceinline__ float rcp_approx(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}

// Shared memory by 32-bit address (a generic pointer is a second register).
__device__ __forceinline__ float4 lds_f4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ int4 lds_i4(uint32_t a) {
  int4 v;
  asm volatile("ld.shared.v4.s32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float lds_f(uint32_t a) {
  float v;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ int lds_flag(uint32_t a) {
  int v;
  asm volatile("ld.volatile.shared.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts_i(uint32_t a, int v) { asm volatile("st.shared.s32 [%0], %1;" ::"r"(a), "r"(v) : "memory"); }
__device__ __forceinline__ void sts_f(uint32_t a, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory"); }
// mbar_wait (decode_stream.cuh) with the abort flag by its shared address.  The word behind the flag says how many of the
// CTA's warps are computing rows again: a wait that sees any begins anew, so that may take as long as the rows' keys do, and
// a wait for something that never comes still ends.
__device__ __forceinline__ void xt_wait(uint32_t bar, uint32_t parity, uint32_t abort_flag, const ExtendTcParams& p) {
  if (lds_flag(abort_flag)) return;
#pragma unroll 1
  for (uint32_t i = 0; i < p.wait_limit; ++i) {
    if (mbar_try_wait(bar, parity)) return;
    if ((i & 1023u) == 1023u) {
      if (lds_flag(abort_flag)) return;
      if (lds_flag(abort_flag + 4u)) i = 0;
    }
  }
  sts_i(abort_flag, 1);
  atomicOr(p.x.err, kErrTimeout);
}
__device__ __forceinline__ void xt_busy(uint32_t busy, int change) {  // one lane
  asm volatile("red.shared.add.s32 [%0], %1;" ::"r"(busy), "r"(change) : "memory");
}

// Codes to operand tiles [2 halves of head_dim][rows][128 B], 16-byte chunks swizzled by row.  A warp takes groups of 8
// rows; a lane holds 16 codes of either half of row lane / 4, quarter lane % 4.  (A store's eight lanes then are two
// neighbouring rows and meet eight different banks; a load's 64 bytes of a row are whole sectors.)
struct XtCodes {
  uint4 c[2];
};
// (Not ld.global.nc: with programmatic launches the kernel may be resident while the one before it stores these rows.)
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p));
  return r;
}
__device__ __forceinline__ void xt_load_codes(XtCodes& r, const uint8_t* base, int row0, int end, int lane) {
  const int row = row0 + (lane >> 2);
  const uint8_t* src = base + (size_t)row * 128 + (lane & 3) * 16;
  r.c[0] = row < end ? ld_stream(src) : make_uint4(0u, 0u, 0u, 0u);
  r.c[1] = row < end ? ld_stream(src + 64) : make_uint4(0u, 0u, 0u, 0u);
}
// Two codes of w (bytes by `sel`) as a bf16 pair: the code's exponent and mantissa bits in bf16's place are the value
// times 2^-120, subnormals included, and the product with 2^120 is exact.
__device__ __forceinline__ uint32_t e4m3x2_to_bf16x2(uint32_t w, uint32_t sel) {
  const uint32_t t = __byte_perm(w, 0u, sel);  // code << 8 in each half
  const uint32_t u = (t & 0x80008000u) | ((t >> 4) & 0x07f007f0u);
  const uint32_t big = 0x7b807b80u;  // 2^120
  const __nv_bfloat162 y = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&u), *reinterpret_cast<const __nv_bfloat162*>(&big));
  return *reinterpret_cast<const uint32_t*>(&y);
}
template <bool BF16>
__device__ __forceinline__ void xt_store_codes(const XtCodes& r, uint8_t* tile, int half_bytes, int row0, int lane) {
  const int row = row0 + (lane >> 2), c0 = 2 * (lane & 3);
  uint8_t* dst = tile + row * 128;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const uint32_t w[4] = {r.c[half].x, r.c[half].y, r.c[half].z, r.c[half].w};
    uint32_t o[8];
    if constexpr (BF16) {
      uint32_t nan = 0u;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        o[2 * u] = e4m3x2_to_bf16x2(w[u], 0x1404u);
        o[2 * u + 1] = e4m3x2_to_bf16x2(w[u], 0x3424u);
        nan |= (w[u] & 0x7f7f7f7fu) + 0x01010101u;
      }
      if (nan & 0x80808080u) {  // a code that is not a number
#pragma unroll
        for (int u = 0; u < 8; ++u) {
          const uint32_t two = (w[u >> 1] >> (16 * (u & 1))) & 0x7f7fu;
          if ((two & 0xffu) == 0x7fu) o[u] |= 0x00007fffu;
          if ((two >> 8) == 0x7fu) o[u] |= 0x7fff0000u;
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        o[2 * u] = e4m3x2_to_half2((unsigned short)(w[u] & 0xffffu));
        o[2 * u + 1] = e4m3x2_to_half2((unsigned short)(w[u] >> 16));
      }
    }
    *reinterpret_cast<uint4*>(dst + half * half_bytes + ((c0 ^ (row & 7)) << 4)) = make_uint4(o[0], o[1], o[2], o[3]);
    *reinterpret_cast<uint4*>(dst + half * half_bytes + (((c0 + 1) ^ (row & 7)) << 4)) = make_uint4(o[4], o[5], o[6], o[7]);
  }
}

// One query row again, by a whole warp, from the visible rows of the piece alone.  redo: lse is computed too (with the
// true maximum); else the caller's is taken.  Returns the output over out_scale, lane = four columns.  For rows whose
// fast result is not finite: a hidden row held something that is not, the weights' sum left its range, or the answer
// is in truth not finite.  d: the piece's words, one per lane.  Far from the tensor cores' rate (512 tokens,
// two KV heads, behind 16000 rows, slopes below zero so that every row comes here: 12 to 17 ms against 0.2), but without limit.
template <bool KV8>
__device__ __forceinline__ float4 xt_row_again(const ExtendTcParams& p, int d, int r, bool redo, float& lse) {
  const ExtendParams& x = p.x;
  auto word = [&](int w) { return __shfl_sync(0xffffffffu, d, w); };
  const int lane = threadIdx.x & 31;
  const int ti = r / x.G, g = r - ti * x.G, h = word(kPwHead), layer = word(kPwLayer), i = word(kPwTok0) + ti;
  const size_t slab = (size_t)word(kPwSlab);
  const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(x.q) + ((size_t)layer * x.total + word(kPwTok) + ti) * x.q_stride + (size_t)(h * x.G + g) * 128;
  const int me = word(kPwSeen) + i;
  const float slope = x.slopes ? x.slopes[h * x.G + g] : 0.f;
  const int kt0 = word(kPwFirst), k0 = kt0 * kPfKeys, end = min((kt0 + word(kPwTiles)) * kPfKeys, word(kPwHeld) + max(i + 1, word(kPwPrefix)));
  auto logit = [&](int j, bool& visible) {
    visible = false;
    if (j >= end) return 0.f;
    const int apart = abs(me - x.pos[slab * x.cap + j]);
    if (x.window > 0 && apart >= x.window) return 0.f;
    visible = true;
    float dot = 0.f;
#pragma unroll 4
    for (int e = 0; e < 128; e += 8) {
      const uint4 qq = *reinterpret_cast<const uint4*>(q + e);
      const size_t at = (slab * x.cap + j) * 128 + e;
      const float4 k0 = ext_row_value4<__nv_bfloat16, KV8>(x.K, at, 1.f), k1 = ext_row_value4<__nv_bfloat16, KV8>(x.K, at + 4, 1.f);
      dot = fmaf(__uint_as_float(qq.x << 16), k0.x, dot);
      dot = fmaf(__uint_as_float(qq.x & 0xffff0000u), k0.y, dot);
      dot = fmaf(__uint_as_float(qq.y << 16), k0.z, dot);
      dot = fmaf(__uint_as_float(qq.y & 0xffff0000u), k0.w, dot);
      dot = fmaf(__uint_as_float(qq.z << 16), k1.x, dot);
      dot = fmaf(__uint_as_float(qq.z & 0xffff0000u), k1.y, dot);
      dot = fmaf(__uint_as_float(qq.w << 16), k1.z, dot);
      dot = fmaf(__uint_as_float(qq.w & 0xffff0000u), k1.w, dot);
    }
    return ext_logit_exact(x, dot, slope, apart);
  };
  if (redo) {
    float m = -CUDART_INF_F, l = 0.f;
    for (int kb = k0; kb < end; kb += 32) {
      bool visible;
      const float y = logit(kb + lane, visible);
      float mx = visible ? y : -CUDART_INF_F;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
      const float mn = fmaxf(m, mx);
      l = l * (m == -CUDART_INF_F ? 0.f : exp2f(m - mn)) + (visible ? exp2f(y - (mn == -CUDART_INF_F ? 0.f : mn)) : 0.f);  // (lane's own sum)
      m = mn;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    lse = m + log2f(l);
  }
  // (Without redo lse is -inf where this part of the item holds no logit above that: it weighs nothing beside the others.  With
  // redo nothing the row sees weighs anything, and the weights are exp2(-inf + inf): NaN.)
  const bool none = !redo && lse == -CUDART_INF_F;
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int kb = k0; kb < end; kb += 32) {
    bool visible;
    const float y = logit(kb + lane, visible);
    const float w = visible && !none ? exp2f(y - lse) : 0.f;
    for (unsigned some = __ballot_sync(0xffffffffu, w != 0.f); some; some &= some - 1) {
      const int kk = __ffs(some) - 1;
      const float wk = __shfl_sync(0xffffffffu, w, kk);
      const float4 v = ext_row_value4<__nv_bfloat16, KV8>(x.V, (slab * x.cap + kb + kk) * 128 + 4 * lane, 1.f);
      acc[0] = fmaf(wk, v.x, acc[0]);
      acc[1] = fmaf(wk, v.y, acc[1]);
      acc[2] = fmaf(wk, v.z, acc[2]);
      acc[3] = fmaf(wk, v.w, acc[3]);
    }
  }
  return make_float4(acc[0], acc[1], acc[2], acc[3]);
}

// Capped logits of 32 columns, c tanh(s / c), in units of the factor it returns.  While every |y| = |s / c| of the warp is
// at most 3/4 -- what a cap is set for -- tanh(y) = y P(y^2) with P the polynomial of degree 5 of the least greatest
// relative error there (3e-8, below a rounding): eight packed operations per two columns on the FMA units.  Beyond,
// tanh(y) = 1 - 2 / (1 + e^(2 y)): two results of the exponentials' unit, which the softmax needs as well and which
// bounds it then.
__device__ __forceinline__ float xt_cap(uint32_t (&sv)[32], const ExtendTcParams& p) {
  float top = 0.f;
#pragma unroll
  for (int c = 0; c < 32; c += 2) top = tc5::f_max3(top, fabsf(__uint_as_float(sv[c])), fabsf(__uint_as_float(sv[c + 1])));
  if (__all_sync(0xffffffffu, top * p.cap_y <= 0.75f)) {
    const uint64_t a2 = tc5::f2_pack(p.cap_y, p.cap_y);
    const float k[6] = {0.999999971f, -0.333329589f, 0.13325406f, -0.0533444308f, 0.0195829087f, -0.00471625728f};
#pragma unroll
    for (int c = 0; c < 32; c += 2) {
      const uint64_t y = tc5::f2_mul(tc5::f2_pack(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), a2), z = tc5::f2_mul(y, y);
      uint64_t t = tc5::f2_pack(k[5], k[5]);
#pragma unroll
      for (int e = 4; e >= 0; --e) t = tc5::f2_fma(t, z, tc5::f2_pack(k[e], k[e]));
      float y0, y1;
      tc5::f2_unpack(tc5::f2_mul(t, y), y0, y1);
      sv[c] = __float_as_uint(y0);
      sv[c + 1] = __float_as_uint(y1);
    }
    return p.cap_log2;
  }
#pragma unroll
  for (int c = 0; c < 32; ++c)
    sv[c] = __float_as_uint(fmaf(-2.f * p.cap_log2, rcp_approx(1.f + fast_exp2(__uint_as_float(sv[c]) * p.cap_arg)), p.cap_log2));
  return 1.f;
}

// x + log2(sum), with the whole part of the logarithm taken out exactly: the approximation is off by 2^-22 of its result,
// which at sums of 2^-33 (a reference with headroom) is 8e-6, and every weight of a mass would carry it.  (Sums that are no
// normal number have no such parts: 0, infinite, or not a number, and so is the result.)
__device__ __forceinline__ float xt_add_log2(float x, float sum) {
  if (!(sum >= 1.17549435e-38f && sum <= 3.4028235e38f)) return x + __log2f(sum);
  const int bits = __float_as_int(sum);
  return (x + (float)((bits >> 23) - 127)) + __log2f(__int_as_float((bits & 0x7fffff) | 0x3f800000));
}

// Joins the parts of the item that begins in CTA blockIdx.x's shares and ends behind them, if there is one: 32 rows per
// block (y), a warp 8 rows x 64 columns, a thread four pieces of four columns of one row.  A part's 128-byte pieces
// are read whole, the output's sectors written whole.  Running maximum and sum over the parts, in the order of the
// list: bound by the latency of three loads (the plan, the list, then the parts, four at once).
constexpr int kXtJoin = 4;
__global__ void __launch_bounds__(256) extend_join_kernel(const __grid_constant__ ExtendTcParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const ExtendParams& x = p.x;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const unsigned share = plan_share0(p.plan, blockIdx.x + 1u) - 1u;
  const int slot = plan_item_of(p.plan, x.seqs.n, share) + (int)blockIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int d = __ldcg(p.plan.words + (size_t)slot * kPlanWords + lane);
  auto word = [&](int w) { return __shfl_sync(0xffffffffu, d, w); };
  const int n_parts = word(kPwParts), rows = word(kPwRows), row = blockIdx.y * 32 + (warp & 3) * 8 + (lane >> 2), c4 = (warp >> 2) * 16 + (lane & 3);
  if (n_parts < 2 || word(kPwBase) != slot) return;  // (an item that began before is another block's)
  if ((int)blockIdx.y * 32 + (warp & 3) * 8 >= rows) return;
  const int tok = word(kPwTok), h = word(kPwHead), layer = word(kPwLayer);
  const int* list = p.plan.words + (size_t)slot * kPlanWords + kPwList;
  int places = lane < n_parts ? __ldcg(list + (size_t)lane * kPlanWords) : 0;  // of the first 32 parts
  const int rr = min(row, rows - 1);
  const size_t piece = (size_t)p.part_rows;
  float M = -CUDART_INF_F, sum = 0.f, acc[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll 1
  for (int k = 0; k < n_parts; k += kXtJoin) {
    if (k > 0 && (k & 31) == 0) places = k + lane < n_parts ? __ldcg(list + (size_t)(k + lane) * kPlanWords) : 0;
    float lk[kXtJoin];
    float4 y[kXtJoin][4];
#pragma unroll
    for (int u = 0; u < kXtJoin; ++u) {  // (behind the last part: the last again, without weight)
      const float* src = p.part + (size_t)__shfl_sync(0xffffffffu, places, min(k + u, n_parts - 1) & 31) * (piece * kXtPartFloats);
      lk[u] = __ldcg(src + 128 * piece + rr);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[u][e] = __ldcg(reinterpret_cast<const float4*>(src) + (size_t)(c4 + 4 * e) * piece + rr);
    }
#pragma unroll
    for (int u = 0; u < kXtJoin; ++u) {
      if (k + u >= n_parts) break;
      const float Mn = fmaxf(M, lk[u]);
      const float keep = M == -CUDART_INF_F ? 0.f : fast_exp2(M - Mn), w = lk[u] == -CUDART_INF_F ? 0.f : fast_exp2(lk[u] - Mn);
      M = Mn;
      sum = fmaf(sum, keep, w);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        acc[4 * e] = fmaf(acc[4 * e], keep, w * y[u][e].x);
        acc[4 * e + 1] = fmaf(acc[4 * e + 1], keep, w * y[u][e].y);
        acc[4 * e + 2] = fmaf(acc[4 * e + 2], keep, w * y[u][e].z);
        acc[4 * e + 3] = fmaf(acc[4 * e + 3], keep, w * y[u][e].w);
      }
    }
  }
  if (row >= rows) return;
  const float f = p.out_scale / sum;
  const int ti = row / x.G;
  __nv_bfloat16* dst = static_cast<__nv_bfloat16*>(x.out) + (((size_t)layer * x.total + tok + ti) * x.Hq + h * x.G + (row - ti * x.G)) * 128 + c4 * 4;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    *reinterpret_cast<uint2*>(dst + 16 * e) = make_uint2(pack_bf16x2(acc[4 * e] * f, acc[4 * e + 1] * f), pack_bf16x2(acc[4 * e + 2] * f, acc[4 * e + 3] * f));
  if (c4 == 0 && x.lse) x.lse[ext_lse_index(x, layer, h, tok) + row] = xt_add_log2(M, sum);
}

// Of this warp's 32 rows (a bit each), those computed again whole (redo: nothing of them is stored yet; the two groups, which
// agree on them, take every other one) and those with elements that are not finite among the group's columns as stored, which
// are replaced.  lse: of each lane's row.  After the stores, for all of a piece in one call: what is rare stays out of the
// way of the rest (called for a block of columns at a time, from their loop, it cost 5 tokens behind 2048 rows 0.7 of 25 us).
template <bool KV8>
__device__ __noinline__ void xt_rows_again(const ExtendTcParams& p, int d, unsigned redo, unsigned bad, float lse, uint32_t busy) {
  const ExtendParams& x = p.x;
  auto word = [&](int w) { return __shfl_sync(0xffffffffu, d, w); };
  const int lane = threadIdx.x & 31, wg = threadIdx.x >> 7, wq = (threadIdx.x >> 5) & 3, h = word(kPwHead), layer = word(kPwLayer), tok = word(kPwTok);
  const bool whole = word(kPwParts) == 1;
  const size_t piece = (size_t)p.part_rows;
  float* part = p.part + (size_t)word(kPwPlace) * (piece * kXtPartFloats);
  __syncwarp();  // (other lanes' stores of a row that is read back here)
  if (lane == 0) xt_busy(busy, 1);
  redo &= wg == 0 ? 0x55555555u : 0xaaaaaaaau;
  for (unsigned left = redo | bad; left; left &= left - 1) {
    const int who = __ffs(left) - 1, row = wq * 32 + who, ti = row / x.G;
    const bool full = (redo >> who) & 1u;
    float row_lse = __shfl_sync(0xffffffffu, lse, who);
    float4 y = xt_row_again<KV8>(p, d, row, full, row_lse);
    if (!full && (lane >> 4) != wg) continue;  // (the other group's columns)
    auto keep = [](float was, float now) { return was * 0.f == 0.f ? was : now; };
    if (whole) {
      uint2* at = reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(x.out) + (((size_t)layer * x.total + tok + ti) * x.Hq + h * x.G + (row - ti * x.G)) * 128 + 4 * lane);
      if constexpr (KV8) y = make_float4(y.x * p.out_scale, y.y * p.out_scale, y.z * p.out_scale, y.w * p.out_scale);
      if (!full) {
        const uint2 o = __ldcg(at);
        y = make_float4(keep(__uint_as_float(o.x << 16), y.x), keep(__uint_as_float(o.x & 0xffff0000u), y.y), keep(__uint_as_float(o.y << 16), y.z),
                        keep(__uint_as_float(o.y & 0xffff0000u), y.w));
      }
      *at = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
      if (full && lane == 0 && x.lse) x.lse[ext_lse_index(x, layer, h, tok) + row] = row_lse;
    } else {
      float4* at = reinterpret_cast<float4*>(part) + (size_t)lane * piece + row;
      if (!full) {
        const float4 o = __ldcg(at);
        y = make_float4(keep(o.x, y.x), keep(o.y, y.y), keep(o.z, y.z), keep(o.w, y.w));
      }
      __stcg(at, y);
      if (full && lane == 0) __stcg(part + 128 * piece + row, row_lse);
    }
  }
  __syncwarp();
  if (lane == 0) xt_busy(busy, -1);
}

// The end of a piece, by the eight softmax warps: a group's 64 columns of the output, or of its part of an item that
// other CTAs share.
template <bool KV8>
__device__ __noinline__ void xt_epilogue(const ExtendTcParams& p, int d, int ord, float ref, float l, uint32_t tO, uint32_t bar0, volatile int* s_abort,
                                         uint8_t* s_out) {
  const ExtendParams& x = p.x;
  auto word = [&](int w) { return __shfl_sync(0xffffffffu, d, w); };
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, wg = warp >> 2, wq = warp & 3;
  const int r = wq * 32 + lane, rows = word(kPwRows), h = word(kPwHead), layer = word(kPwLayer), tok = word(kPwTok);
  const bool whole = word(kPwParts) == 1;
  const uint32_t abort_flag = bar0 + 124u, busy = bar0 + 128u;
  xt_wait(bar0 + 8 * 12, (uint32_t)(ord & 1), abort_flag, p);
  tc5::fence_after_sync();
  if (wq * 32 >= rows) {  // no query in this warp's rows
    mbar_arrive(bar0 + 8 * 7);
    return;
  }
  const uint32_t g_inv = 65536u / (uint32_t)x.G + 1u;
  uint8_t* stage = s_out + warp * kXtStageBytes;
  const bool mine = r < rows;
  const size_t piece = (size_t)p.part_rows;
  float* part = p.part + (size_t)word(kPwPlace) * (piece * kXtPartFloats);
  // Out of range, or not a number; or the reference tiles held nothing above -inf, so that the sum has no reference (or the row
  // of a whole item no sum: it sees itself, so all it sees is -inf).
  const bool gave_up = __any_sync(0xffffffffu, *s_abort != 0);  // (nothing is computed again then, nor stored)
  const bool redo = mine && !gave_up && (!(l < kXtSumMax) || (ref == -CUDART_INF_F && (whole || l > 0.f)));
  const float lse = l > 0.f ? xt_add_log2(ref, l) : -CUDART_INF_F;
  const float f = l > 0.f ? 1.f / l : 0.f;
  __nv_bfloat16* obase = static_cast<__nv_bfloat16*>(x.out) + (((size_t)layer * x.total + tok) * x.Hq + h * x.G) * 128;
  const uint32_t t_row = tO + ((uint32_t)(wq * 32) << 16);
  const unsigned redone = __ballot_sync(0xffffffffu, redo);
  bool finite = true;  // this row's columns here are
#pragma unroll 1
  for (int c0 = 64 * wg; c0 < 64 * wg + 64; c0 += 32) {
    uint32_t o[32];
    tc5::tmem_ld32(t_row + (uint32_t)c0, o);
    tc5::tmem_wait_ld();
    if (c0 == 64 * wg + 32) {
      tc5::fence_before_sync();
      mbar_arrive(bar0 + 8 * 7);  // O may be written again
    }
    const uint64_t f2 = tc5::f2_pack(f, f);
    uint64_t probe[2] = {0ull, 0ull};  // 0 * finite = 0
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint64_t y = tc5::f2_mul(tc5::f2_pack(__uint_as_float(o[2 * e]), __uint_as_float(o[2 * e + 1])), f2);
      probe[e & 1] = tc5::f2_fma(y, 0ull, probe[e & 1]);
      float y0, y1;
      tc5::f2_unpack(y, y0, y1);
      o[2 * e] = __float_as_uint(y0);
      o[2 * e + 1] = __float_as_uint(y1);
    }
    float p0, p1;
    tc5::f2_unpack(tc5::f2_add(probe[0], probe[1]), p0, p1);
    finite = finite && p0 + p1 == 0.f;
    if (whole) {
      // rounded, through the warp's staging tile [32 rows][64 B] (16-byte chunks swizzled), so that the stores are 64-byte
      // pieces of rows
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t y[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float y0 = __uint_as_float(o[8 * e + 2 * u]), y1 = __uint_as_float(o[8 * e + 2 * u + 1]);
          if constexpr (KV8) {
            y0 *= p.out_scale;
            y1 *= p.out_scale;
          }
          y[u] = pack_bf16x2(y0, y1);
        }
        *reinterpret_cast<uint4*>(stage + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
      }
      __syncwarp();
      const bool store = *s_abort == 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 8 * i + (lane >> 2), chunk = lane & 3;
        const uint4 v = *reinterpret_cast<const uint4*>(stage + row * 64 + ((chunk ^ ((row >> 1) & 3)) << 4));
        const int rr = wq * 32 + row, ti = (int)((uint32_t)rr * g_inv >> 16);
        if (rr < rows && store && !((redone >> row) & 1u)) *reinterpret_cast<uint4*>(obase + (ti * x.Hq + (rr - ti * x.G)) * 128 + c0 + chunk * 8) = v;
      }
      __syncwarp();
    } else if (mine && !redo && !*s_abort) {
      float4* dst = reinterpret_cast<float4*>(part) + (size_t)c0 / 4 * piece + r;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        __stcg(dst + e * piece,
               make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]), __uint_as_float(o[4 * e + 3])));
    }
  }
  if (wg == 0 && mine && !redo && !*s_abort) {
    if (!whole) __stcg(part + 128 * piece + r, lse);
    else if (x.lse) x.lse[ext_lse_index(x, layer, h, tok) + r] = lse;
  }
  // Elements of the others that are not finite: something V holds, seen or hidden.
  const unsigned bad = __ballot_sync(0xffffffffu, mine && !redo && !gave_up && !finite);
  if (redone | bad) xt_rows_again<KV8>(p, d, redone, bad, lse, busy);
}

template <bool KV8, bool MODS>
__global__ void __launch_bounds__((XtShape<KV8, MODS>::kThreads), 2)
extend_tc_kernel(const __grid_constant__ ExtendTcParams p, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                 const __grid_constant__ CUtensorMap tmV) {
  extern __shared__ __align__(1024) uint8_t pf_smem[];
  uint8_t* sm = pf_smem;
  const uint32_t sQ = smem_u32(sm);                       // [2 halves of head_dim][128 rows][128 B]
  const uint32_t sK = sQ + kPfQBytes;                     // [2 stages][2 halves][64 rows][128 B]
  const uint32_t sV = sK + 2 * kPfKvBytes;                // the same
  uint8_t* s_out = sm + kPfQBytes + 4 * kPfKvBytes;       // [8 softmax warps][2 KB]
  uint64_t* bars = reinterpret_cast<uint64_t*>(s_out + 8 * kXtStageBytes);
  // barriers: 0 Q, 1-2 K stages filled, 3-4 V stages filled, 5-6 S buffers complete, 7 O has been read, 8-9 P written (per S
  // buffer), 10-11 V stages and P read, 12 the piece's last O += P V complete, 13-14 drain
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 15);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  const ExtendParams& x = p.x;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  constexpr bool kLoaders = XtShape<KV8, MODS>::kLoaders;
  constexpr int kSWarp = kLoaders ? 10 : 8, kOWarp = kSWarp + 1;  // the warps that issue S and O
  if (tid == 0) {
    for (int i = 0; i < 15; ++i) mbar_init(bar(i), i == 7 ? 2 * kXtRows : (i == 8 || i == 9) ? kXtRows : KV8 && (i == 1 || i == 2) ? 2 : 1);
    *s_abort = 0;
    s_abort[1] = 0;  // (warps that compute rows again)
    if ((smem_u32(sm) & 1023u) != 0u) {
      atomicOr(x.err, kErrStreamBounds);
      *s_abort = 1;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == kSWarp) {
    tc5::tmem_alloc(smem_u32(s_tmem), kPfTmemCols);
    tc5::tmem_relinquish();
  }
  if (tid == kOWarp * 32) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmQ)) : "memory");
    if constexpr (!KV8) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmK)) : "memory");
      asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tmV)) : "memory");
    }
  }
  // This CTA's pieces: the items of its first and its last share (lanes 0 and 1), slots side by side.
  const unsigned share = lane == 0 ? plan_share0(p.plan, blockIdx.x) : plan_share0(p.plan, blockIdx.x + 1u) - 1u;
  const int item = plan_item_of(p.plan, x.seqs.n, share) + (int)blockIdx.x;
  int slot = __shfl_sync(0xffffffffu, item, 0);
  const int slot_end = __shfl_sync(0xffffffffu, item, 1) + 1;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (the next kernel finds room when CTAs of this one end, and waits for all)
  // The storing kernel may still be running; everything below waits until it has completed.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int d = __ldcg(p.plan.words + (size_t)slot * kPlanWords + lane);  // the piece's words, one per lane
  tc5::fence_before_sync();
  __syncthreads();
  tc5::fence_after_sync();
  const uint32_t tmem = *s_tmem;
  const uint32_t tS0 = tmem, tO = tmem + 128;  // S buffer b at column 64 b
  auto word = [&](int w) { return __shfl_sync(0xffffffffu, d, w); };
  // the next piece that holds any key tile; its words are asked for when a piece begins
  int d_next = 0;
  auto ask_next = [&]() {
    if (slot + 1 < slot_end) d_next = __ldcg(p.plan.words + (size_t)(slot + 1) * kPlanWords + lane);
  };
  auto go_next = [&]() {
    ++slot;
    d = d_next;
  };
  auto load_q = [&]() {  // the piece's queries
    const int tok = word(kPwLayer) * x.total + word(kPwTok), head = word(kPwHead) * x.G;
    if (tc5::elect_one()) {
      mbar_arrive_expect_tx(bar(0), 256u * (uint32_t)(x.G * p.plan.tokens_per_tile));
      pf_tma_load(sQ, &tmQ, 0, head, tok, bar(0));
      pf_tma_load(sQ + kPfQBytes / 2, &tmQ, 64, head, tok, bar(0));
    }
    __syncwarp();
  };

  auto load_tile = [&](bool k, int g, int row, int slab) {  // a K or V tile by TMA into the stage of tile g
    if (tc5::elect_one()) {
      const uint32_t dst = (k ? sK : sV) + (uint32_t)(g & 1) * kPfKvBytes, bb = bar((k ? 1 : 3) + (g & 1));
      const CUtensorMap* tm = k ? &tmK : &tmV;
      mbar_arrive_expect_tx(bb, kPfKvBytes);
      pf_tma_load(dst, tm, 0, row, slab, bb);
      pf_tma_load(dst + kPfKvBytes / 2, tm, 64, row, slab, bb);
    }
    __syncwarp();
  };

  if (kLoaders && (warp == 8 || warp == 9)) {
    // ================= the warps that load: 8 Q and K, 9 V; 8-bit rows: 8 Q and half of K, 9 the other half =================
    if (lane == 0 && *reinterpret_cast<volatile int*>(p.stop) != 0) *s_abort = 1;
    __syncwarp();
    int g = 0;
    for (; slot < slot_end && !*s_abort; go_next()) {
      ask_next();
      const int nkt = word(kPwTiles), kt_new = word(kPwFirst) + nkt - 1, slab = word(kPwSlab), end = word(kPwHeld) + word(kPwNew);
      // 8-bit rows: this warp's 32 rows of a tile, eight at a time, each eight a whole tile ahead in registers
      XtCodes codes[4];
      const uint8_t* src = KV8 ? static_cast<const uint8_t*>(x.K) + (size_t)slab * x.cap * 128 : nullptr;
      const int sub = 32 * (warp & 1);
      if constexpr (KV8) {
        if (nkt > 0) {
#pragma unroll
          for (int i = 0; i < 4; ++i) xt_load_codes(codes[i], src, kt_new * kPfKeys + sub + 8 * i, end, lane);
        }
      }
      for (int j = 0; j < nkt; ++j, ++g) {
        // The piece's Q, once the last S of the piece before has been computed from its own; a K stage is filled again when
        // S of tile g - 2 has read it, a V stage when O += P V of tile g - 2 has.
        const bool new_q = warp == 8 && j == 0;
        const int done = new_q ? g - 1 : g - 2, freed = KV8 || warp == 8 ? 5 : 10;
        if (done >= 0) xt_wait(bar(freed + (done & 1)), (uint32_t)((done >> 1) & 1), bar0 + 124u, p);
        __syncwarp();
        if (*s_abort) break;
        if (new_q) load_q();
        if constexpr (KV8) {
          uint8_t* tile = sm + kPfQBytes + (uint32_t)(g & 1) * kPfKvBytes;
          const int k0 = (kt_new - j - 1) * kPfKeys + sub;
          // (four tiles further on towards the older rows: asked into L2)
          if (lane == 0 && j + 4 < nkt)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(src + (size_t)(k0 - 3 * kPfKeys) * 128), "r"(32 * 128) : "memory");
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            xt_store_codes<false>(codes[i], tile, kPfKvBytes / 2, sub + 8 * i, lane);
            if (j + 1 < nkt) xt_load_codes(codes[i], src, k0 + 8 * i, end, lane);
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(1 + (g & 1)));
          __syncwarp();
        } else {
          load_tile(warp == 8, g, (kt_new - j) * kPfKeys, slab);
        }
      }
    }
    if (*s_abort && lane == 0) {
      // Something gave up: a bounded time for the loads this warp started (see prefill_attn.cuh).
      atomicOr(p.stop, 1);
      for (int i = warp == 8 ? 0 : 3; i < (warp == 8 ? (KV8 ? 1 : 3) : (KV8 ? 3 : 5)); ++i)
        for (uint32_t ph = 0; ph < 2; ++ph)
          for (uint32_t w = 0; w < (1u << 16); ++w)
            if (mbar_try_wait(bar(i), ph)) break;
    }
  } else if (warp == kSWarp || warp == kOWarp) {
    // ================= the warps that issue S = Q K^T and O += P V (and load, where no others do) =================
    if (lane == 0 && *reinterpret_cast<volatile int*>(p.stop) != 0) *s_abort = 1;
    __syncwarp();
    auto issue = [&](auto which) {
      constexpr bool is_s = decltype(which)::value;
      constexpr uint32_t idesc = is_s ? (KV8 ? tc5::idesc_f16_f32(kXtRows, kPfKeys, 0, 0) : tc5::idesc_bf16_f32(kXtRows, kPfKeys, 0, 0))
                                      : tc5::idesc_bf16_f32(kXtRows, 128, 0, 1);
      const uint64_t dQ = tc5::smem_desc_sw128(sQ, 16, 1024);
      const uint64_t dKV = is_s ? tc5::smem_desc_sw128(sK, 16, 1024) : tc5::smem_desc_sw128(sV, kPfKvBytes / 2, 1024);
      int g = 0, ord = 0, j = 0, nkt = 0;
      auto find = [&]() {  // the next piece that holds any key tile
        while (slot < slot_end) {
          ask_next();
          nkt = word(kPwTiles);
          if (nkt > 0) break;
          go_next();
        }
        j = 0;
      };
      // Loads run two tiles ahead of the products, over the pieces' words a second time.
      int l_slot = slot, l_d = d, l_j = 0, l_nkt = kLoaders ? 0 : word(kPwTiles);
      auto load = [&](int gl) {  // K (or V) of tile gl, if there is one
        while (l_slot < slot_end && l_j == l_nkt) {
          if (++l_slot < slot_end) {
            l_d = __ldcg(p.plan.words + (size_t)l_slot * kPlanWords + lane);
            l_nkt = __shfl_sync(0xffffffffu, l_d, kPwTiles);
            l_j = 0;
          }
        }
        if (l_slot >= slot_end) return;
        const int row = (__shfl_sync(0xffffffffu, l_d, kPwFirst) + l_nkt - 1 - l_j) * kPfKeys;
        ++l_j;
        load_tile(is_s, gl, row, __shfl_sync(0xffffffffu, l_d, kPwSlab));
      };
      find();
      if constexpr (!kLoaders) {
        if (!*s_abort) {
          if (is_s && slot < slot_end) load_q();
          load(0);
          load(1);
        }
      }
      while (slot < slot_end && !*s_abort) {
        const int st = g & 1;
        if constexpr (is_s) {
          xt_wait(bar(1 + st), (uint32_t)((g >> 1) & 1), bar0 + 124u, p);
          // S of tile g overwrites the columns P of tile g - 2 is read from
          if (g >= 2) xt_wait(bar(10 + st), (uint32_t)(((g - 2) >> 1) & 1), bar0 + 124u, p);
          if (j == 0) xt_wait(bar(0), (uint32_t)(ord & 1), bar0 + 124u, p);
        } else {
          if constexpr (!KV8) xt_wait(bar(3 + st), (uint32_t)((g >> 1) & 1), bar0 + 124u, p);  // (8-bit rows: written before P)
          xt_wait(bar(8 + st), (uint32_t)((g >> 1) & 1), bar0 + 124u, p);
          if (j == 0 && ord > 0) xt_wait(bar(7), (uint32_t)((ord - 1) & 1), bar0 + 124u, p);  // O of the piece before has been read
        }
        __syncwarp();
        tc5::fence_after_sync();
        if (*s_abort) break;
        const uint64_t dg = dKV + (uint64_t)((uint32_t)st * (kPfKvBytes >> 4));
        if (tc5::elect_one()) {
          if constexpr (is_s) {
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              tc5::mma_bf16_ss(tS0 + 64u * (uint32_t)st, dQ + (uint64_t)((kk >> 2) * (kPfQBytes >> 5) + (kk & 3) * 2),
                               dg + (uint64_t)((kk >> 2) * (kPfKvBytes >> 5) + (kk & 3) * 2), idesc, kk > 0);
            tc5::mma_commit(bar(5 + st));
          } else {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)  // 16 keys per step: 8 columns of P (over S buffer g & 1), two 8-row groups of V
              tc5::mma_bf16_ts(tO, tS0 + 64u * (uint32_t)st + 8u * (uint32_t)kk, dg + (uint64_t)(kk * 128), idesc, (j > 0 || kk > 0) ? 1u : 0u);
            tc5::mma_commit(bar(10 + st));
            if (j == nkt - 1) tc5::mma_commit(bar(12));
          }
        }
        __syncwarp();
        const bool last = ++j == nkt;
        if constexpr (!kLoaders) {
          if (l_slot < slot_end || last) {  // the stage of this tile (and, with a piece's last S, Q) is free when its product is done
            xt_wait(bar((is_s ? 5 : 10) + st), (uint32_t)((g >> 1) & 1), bar0 + 124u, p);
            __syncwarp();
            if (*s_abort) break;
            load(g + 2);
          }
        }
        ++g;
        if (last) {
          ++ord;
          go_next();
          find();
          if constexpr (!kLoaders) {
            if (is_s && slot < slot_end) load_q();
          }
        }
      }
      if (*s_abort) {
        // Something gave up: a bounded time for the loads this warp started and the MMAs already issued (see prefill_attn.cuh)
        if (lane == 0) {
          atomicOr(p.stop, 1);
          if constexpr (!kLoaders)
            for (int i = is_s ? 0 : 3; i < (is_s ? 3 : 5); ++i)
              for (uint32_t ph = 0; ph < 2; ++ph)
                for (uint32_t w = 0; w < (1u << 16); ++w)
                  if (mbar_try_wait(bar(i), ph)) break;
        }
        __syncwarp();
        if (tc5::elect_one()) {
          tc5::mma_commit(bar(is_s ? 14 : 13));
          for (uint32_t w = 0; w < kPfSpinLimit; ++w)
            if (mbar_try_wait(bar(is_s ? 14 : 13), 0u)) break;
        }
      }
    };
    if (warp == kSWarp) issue(std::true_type{});
    else issue(std::false_type{});
  } else {
    // ================= softmax warps: thread = query row = tensor-memory lane =================
    const int wg = warp >> 2, wq = warp & 3;              // group; warp within it (its lanes of tensor memory)
    const uint32_t stage = smem_u32(s_out) + (uint32_t)warp * kXtStageBytes;
    const uint32_t abort_flag = bar0 + 124u;
    const uint32_t t_row = tS0 + ((uint32_t)(wq * 32) << 16);
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;" ::"r"(2 + wq) : "memory"); };
    int g0 = 0, ord = 0;  // flat index of the piece's first tile, piece
    for (; slot < slot_end; go_next()) {
      ask_next();
      const int nkt = word(kPwTiles);
      if (nkt == 0) continue;
      const int kt_new = word(kPwFirst) + nkt - 1;  // its newest tile
      const int rows = word(kPwRows), held = word(kPwHeld), i0 = word(kPwTok0), prefix = word(kPwPrefix);
      const bool live = wq * 32 < rows;
      const int r = min(wq * 32 + lane, rows - 1);  // (a lane without a query repeats the last row's visibility)
      const int ti = i0 + r / x.G;
      const int lim = held + max(ti + 1, prefix);   // rows [0, lim) are visible
      // Tiles that some token of the query tile does not see whole, and one more, are the first group's: after them every row
      // that sees anything has its reference.  (With a window a token of a prefix may see only rows around its own: down to those.)
      const int whole_to = held + (MODS && x.window > 0 ? i0 : max(i0 + 1, prefix) - 1);
      const int ramp = min(nkt, max(0, kt_new - whole_to / kPfKeys) + 1);
      const int* pos_row = nullptr;
      int tot = 0;
      float slope = 0.f;
      if constexpr (MODS) {
        tot = word(kPwSeen);
        pos_row = x.pos + (size_t)word(kPwSlab) * x.cap;
        if (x.slopes) slope = x.slopes[word(kPwHead) * x.G + r % x.G] * 1.4426950408889634f;
      }
      const uint8_t* v_codes = KV8 ? static_cast<const uint8_t*>(x.V) + (size_t)word(kPwSlab) * x.cap * 128 : nullptr;
      const int end = held + word(kPwNew);
      float ref = -CUDART_INF_F, l = 0.f;
      int j = wg == 0 ? 0 : ramp;
      if (wg == 1) {  // the reference comes from the first group's first tiles
        pair_sync();
        ref = lds_f(smem_u32(s_out) + (uint32_t)(warp ^ 4) * kXtStageBytes + 512u + 4u * lane);  // (of the warp with the same rows)
      }
#pragma unroll 1
      while (j < nkt) {
        // One tile: S of flat tile g to P, a chunk of columns at a time.  In the ramp part of the tile may be hidden and
        // the reference may not be set yet: S is read twice.
        const bool in_ramp = j < ramp;
        const int g = g0 + j, key0 = (kt_new - j) * kPfKeys;
        const uint32_t ts = t_row + 64u * (uint32_t)(g & 1);
        int pos_a = 0, pos_b = 0;
        if constexpr (MODS) {  // positions, the chunk's first token being 0: two per lane
          pos_a = pos_row[min(key0 + lane, x.cap - 1)] - tot;
          pos_b = pos_row[min(key0 + 32 + lane, x.cap - 1)] - tot;
        }
        XtCodes vc[2];
        if constexpr (KV8) {  // this warp's 16 rows of V
          xt_load_codes(vc[0], v_codes, key0 + 16 * wq, end, lane);
          xt_load_codes(vc[1], v_codes, key0 + 16 * wq + 8, end, lane);
          if (lane == 0 && j + 4 < nkt)
            asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(v_codes + (size_t)(key0 + 16 * wq - 4 * kPfKeys) * 128), "r"(16 * 128) : "memory");
        }
        auto widen_v = [&]() {
          uint8_t* vt = sm + kPfQBytes + (2 + (uint32_t)(g & 1)) * kPfKvBytes;
          xt_store_codes<true>(vc[0], vt, kPfKvBytes / 2, 16 * wq, lane);
          xt_store_codes<true>(vc[1], vt, kPfKvBytes / 2, 16 * wq + 8, lane);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        };
        // 8-bit rows: V goes to its stage while S is computed, once O += P V of tile g - 2 has read it (4096 behind 4096: 550 -> 540 us);
        // with caps, biases and windows after it, as the two waits cost more than they hide (a capped step of 64: 93 against 98 us).
        if constexpr (KV8 && !MODS) {
          if (g >= 2) xt_wait(bar(10 + (g & 1)), (uint32_t)(((g - 2) >> 1) & 1), abort_flag, p);
          widen_v();
        }
        xt_wait(bar(5 + (g & 1)), (uint32_t)((g >> 1) & 1), abort_flag, p);  // S of this tile is complete
        tc5::fence_after_sync();
        if constexpr (KV8 && MODS) widen_v();  // (S of this tile was issued after O += P V of tile g - 2 had read the stage)
        if (live) {
          constexpr int CH = 32;
          bool border = false, beside = false;
          float at = 0.f;                                       // this row's token
          // (the staging tile: positions counted from the tile's newest row, [64] as integers and [64] as floats)
          int me = 0;
          if constexpr (MODS) {
            // From the newest: a token is at most 64 positions closer to it than to any row it sees, so both terms of a
            // bias are about as small as the bias.  (From the first, which may have survived evictions from far back, a recent
            // row's bias would be the difference of two large products.)
            const int last = min(kPfKeys, end - key0) - 1, p0 = __shfl_sync(0xffffffffu, last < 32 ? pos_a : pos_b, last & 31);
            __syncwarp();
            sts_i(stage + 4u * lane, pos_a - p0);
            sts_i(stage + 128u + 4u * lane, pos_b - p0);
            sts_f(stage + 256u + 4u * lane, (float)(pos_a - p0));
            sts_f(stage + 384u + 4u * lane, (float)(pos_b - p0));
            me = ti - p0;
            at = (float)me;
            const bool fresh = key0 + kPfKeys > held;  // the tile holds rows of the chunk
            // the tile's first position against the warp's last token (in tiles with rows of the chunk: always compared)
            border = x.window > 0 && (fresh || __shfl_sync(0xffffffffu, ti, 31) - __shfl_sync(0xffffffffu, pos_a, 0) >= x.window);
            beside = fresh && prefix > 0;  // rows of later positions may be visible
            __syncwarp();
          }
          uint64_t sum2[2] = {0ull, 0ull};  // two chains of (even, odd) column sums
          // (a row's reference comes from the first half of the first tile it sees: the headroom is for all others)
#pragma unroll 1
          for (int step = in_ramp && __any_sync(0xffffffffu, ref == -CUDART_INF_F) ? -1 : 0; step < kPfKeys / CH; ++step) {
            const int hb = step < 0 ? 0 : step * CH;
            uint32_t sv[CH];
            tc5::tmem_ld32(ts + (uint32_t)hb, sv);
            tc5::tmem_wait_ld();
            float scale_log2 = p.scale_log2;  // logits in base-2 units: scaled in the exponent's multiply-add, or with a bias before it
            if constexpr (MODS) {
              if (x.cap_logit > 0.f) scale_log2 = xt_cap(sv, p);
              const float scale = scale_log2;
              if (x.slopes) scale_log2 = 1.f;
              const uint64_t scale2 = tc5::f2_pack(scale, scale);
              if (!x.slopes) {
              } else if (beside) {
#pragma unroll
                for (int c = 0; c < CH; ++c) sv[c] = __float_as_uint(fmaf(__uint_as_float(sv[c]), scale, -slope * fabsf(at - lds_f(stage + 256u + 4u * (uint32_t)(hb + c)))));
              } else {  // - slope (me - pos) = slope pos - slope me, both counted from the tile's newest row
                const uint64_t slope2 = tc5::f2_pack(slope, slope), base2 = tc5::f2_pack(-slope * at, -slope * at);
#pragma unroll
                for (int c = 0; c < CH; c += 4) {
                  const float4 y = lds_f4(stage + 256u + 4u * (uint32_t)(hb + c));
                  float x0, x1, x2, x3;
                  tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), scale2,
                                             tc5::f2_fma(tc5::f2_pack(y.x, y.y), slope2, base2)), x0, x1);
                  tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[c + 2]), __uint_as_float(sv[c + 3])), scale2,
                                             tc5::f2_fma(tc5::f2_pack(y.z, y.w), slope2, base2)), x2, x3);
                  sv[c] = __float_as_uint(x0);
                  sv[c + 1] = __float_as_uint(x1);
                  sv[c + 2] = __float_as_uint(x2);
                  sv[c + 3] = __float_as_uint(x3);
                }
              }
              if (border) {
#pragma unroll
                for (int c = 0; c < CH; c += 4) {
                  const int4 y = lds_i4(stage + 4u * (uint32_t)(hb + c));
                  if (abs(me - y.x) >= x.window) sv[c] = 0xff800000u;  // -inf
                  if (abs(me - y.y) >= x.window) sv[c + 1] = 0xff800000u;
                  if (abs(me - y.z) >= x.window) sv[c + 2] = 0xff800000u;
                  if (abs(me - y.w) >= x.window) sv[c + 3] = 0xff800000u;
                }
              }
            }
            if (in_ramp) {
              const int cv = lim - key0 - hb;  // visible columns of the chunk
#pragma unroll
              for (int c = 0; c < CH; ++c)
                if (c >= cv) sv[c] = 0xff800000u;
              // A row with a window may see nothing in the first half and something in the second.
              if (ref == -CUDART_INF_F) {
                float mx4[4] = {-CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F, -CUDART_INF_F};
#pragma unroll
                for (int c = 0; c < CH; c += 8)
#pragma unroll
                  for (int u = 0; u < 4; ++u) mx4[u] = tc5::f_max3(mx4[u], __uint_as_float(sv[c + u]), __uint_as_float(sv[c + 4 + u]));
                ref = tc5::f_max3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]) * scale_log2 + kXtHeadroom;
              }
              if (step < 0) continue;
            }
            const float neg = ref == -CUDART_INF_F ? 0.f : -ref;
            const uint64_t scale2 = tc5::f2_pack(scale_log2, scale_log2), neg2 = tc5::f2_pack(neg, neg);
            uint32_t pk[CH / 2];
#pragma unroll
            for (int c = 0; c < CH / 2; ++c) {
              float x0, x1;
              tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[2 * c]), __uint_as_float(sv[2 * c + 1])), scale2, neg2), x0, x1);
              const float a0 = fast_exp2(x0), a1 = fast_exp2(x1);
              sum2[c & 1] = tc5::f2_add(sum2[c & 1], tc5::f2_pack(a0, a1));
              pk[c] = pack_bf16x2(a0, a1);
            }
            tc5::tmem_st16(ts + (uint32_t)(hb / 2), pk);  // (over columns of S that have been read)
          }
          float e, o;
          tc5::f2_unpack(tc5::f2_add(sum2[0], sum2[1]), e, o);
          l += e + o;
          tc5::tmem_wait_st();
        }
        tc5::fence_before_sync();
        mbar_arrive(bar(8 + (g & 1)));
        if (wg == 1) {
          j += 2;
        } else if (++j == ramp) {
          sts_f(stage + 512u + 4u * lane, ref);
          pair_sync();
          ++j;
        } else if (j > ramp) {
          ++j;
        }
      }
      g0 += nkt;
      // the other group's share of the row's sum
      sts_f(stage + 640u + 4u * lane, l);
      pair_sync();
      const float l_other = lds_f(smem_u32(s_out) + (uint32_t)(warp ^ 4) * kXtStageBytes + 640u + 4u * lane);
      l = wg == 0 ? l + l_other : l_other + l;
      pair_sync();
      xt_epilogue<KV8>(p, d, ord, ref, l, tO, bar0, s_abort, s_out);
      ++ord;
    }
  }
  tc5::fence_before_sync();
  __syncthreads();
  if (warp == kSWarp) tc5::tmem_dealloc(tmem, kPfTmemCols);
}

// extend_mass_tc_kernel: mass_j = sum over the chunk's tokens i and the group's heads of exp2(x_ij - lse_i).
// The products are taken the other way round -- M = 128 keys, N = 128 query rows -- so that thread = key = tensor-
// memory lane: the sum over the queries stays in one register, needs no exchange between lanes and no atomics, and
// exactly one thread writes a row.  A work item = 256 rows of one slab, 128 for each of two groups of four warps, against
// the query rows that see any of them, in steps of 128; where the items are fewer than the CTAs the steps of each are
// cut into parts, whose sums the last part to finish adds in order.  Persistent CTAs, two per SM; K 64 KB, Q 32 KB, one S
// of 128 columns per group: while a group's S is made the other three groups of the SM compute.  (With 128 keys per item
// the Q tiles, read again from L2 for every item, bounded it: 1.25 times as long.  With steps of 64 query rows in two buffers
// per group the products did: 57 cycles instead of 64 for half the work, as the keys' 4 KB are read all the same.)
// Four ragged sequences of 3782 new tokens behind 2000 to 6000 rows: 215 us, 0.57 PFLOP/s of products, the exponentials' unit
// busy for 0.66 of the time; what is left is unlike parts (0.15) and the waits of a part's beginning and end.
constexpr int kXmThreads = 320;
constexpr int kXmKeys = 128;                      // keys per group
constexpr int kXmItemKeys = 2 * kXmKeys;
constexpr int kXmRows = kXtRows;                       // query rows per step
constexpr int kXmKBytes = kXmKeys * 256;
constexpr int kXmQBytes = kXmRows * 256;
constexpr int kXmWarpFloats = 2 * kXmRows;                // per compute warp: a step's additive constants, its columns' negated slopes
constexpr int kXmSmemBytes = 2 * kXmKBytes + kXmQBytes + 192 + (8 * kXmWarpFloats + kXmRows) * 4 + (2 * kExtSeqs + 1) * 4 + 12;
constexpr uint32_t kXmTmemCols = 256;

struct XmCursor {
  int it, ord;        // position in this CTA's list; items with steps before it
  int lo, n_step;     // first query tile, query tiles
  int s, layer, h, n, t, k0;
  int item, part;
};

struct XmShared {
  const int* n;      // rows held by each sequence
  const int* item0;  // first (sequence, key tile) of each sequence
  int n_work, parts;
};

__device__ __forceinline__ void xm_seek(XmCursor& c, int it, int n_items, const ExtendTcParams& p, const XmShared& sh, bool skip_empty) {
  const int tps = kXmRows / p.x.G;  // tokens per step
  for (; it < n_items; ++it) {
    const int w = (int)blockIdx.x + it * (int)gridDim.x;
    const int up = w / p.plan.lh, lh = w - up * p.plan.lh;
    const int u = sh.parts == 1 ? up : up / sh.parts;
    c.part = up - u * sh.parts;
    c.item = u * p.plan.lh + lh;
    c.s = ext_find(sh.item0, p.x.seqs.n, u);
    c.n = sh.n[c.s];
    c.t = p.x.seqs.tok0[c.s + 1] - p.x.seqs.tok0[c.s];
    c.k0 = (u - sh.item0[c.s]) * kXmItemKeys;
    c.layer = p.x.n_layers == 1 ? 0 : lh / p.x.Hkv;
    c.h = lh - c.layer * p.x.Hkv;
    int lo = c.k0 < c.n + p.x.seqs.prefix[c.s] ? 0 : (c.k0 - c.n) / tps;
    int hi = (c.t + tps - 1) / tps;
    if (p.x.window > 0) {  // a token is at least as many positions behind a row as it is rows behind it
      const long long last = (long long)p.x.window + c.k0 + kXmItemKeys - 1 - c.n;  // tokens from here on see none of the rows
      hi = last <= 0 ? 0 : (int)min((long long)hi, (last + tps - 1) / tps);
    }
    hi = max(lo, hi);
    if (sh.parts > 1) {
      const int steps = hi - lo, per = (steps + sh.parts - 1) / sh.parts;
      lo = min(hi, lo + c.part * per);
      hi = min(hi, lo + per);
    }
    c.lo = lo;
    c.n_step = hi - lo;
    if (c.n_step > 0 || !skip_empty) break;
  }
  c.it = it;
}

template <bool KV8, bool MODS>
__global__ void __launch_bounds__(kXmThreads, 2)
extend_mass_tc_kernel(const __grid_constant__ ExtendTcParams p, const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK) {
  extern __shared__ __align__(1024) uint8_t pf_smem[];
  uint8_t* sm = pf_smem;
  const uint32_t sK = smem_u32(sm);             // [2 groups][2 halves of head_dim][128 rows][128 B]
  const uint32_t sQ = sK + 2 * kXmKBytes;       // [2 halves][128 rows][128 B]
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + 2 * kXmKBytes + kXmQBytes);
  // barriers: 0 K filled, 1 Q filled, 2-3 a group's S complete, 4-5 a group's S read, 6 K read, 7 drain
  const uint32_t bar0 = smem_u32(bars);
  auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
  uint32_t* s_tmem = reinterpret_cast<uint32_t*>(bars + 15);
  volatile int* s_abort = reinterpret_cast<volatile int*>(s_tmem + 1);
  int* s_flag = reinterpret_cast<int*>(s_tmem + 3);  // (the word between stays 0: no rows are computed again here, see xt_wait)
  float* s_warp = reinterpret_cast<float*>(bars + 24);
  float* s_tok = s_warp + 8 * kXmWarpFloats;    // token of a column within its step
  int* s_n = reinterpret_cast<int*>(s_tok + kXmRows);
  int* s_item0 = s_n + kExtSeqs;
  const ExtendParams& x = p.x;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int tps = kXmRows / x.G;

  if (tid == 0) {
    for (int i = 0; i < 8; ++i) mbar_init(bar(i), i == 0 && KV8 ? 8 : i == 4 || i == 5 ? kXmKeys : 1);
    *s_abort = 0;
    s_abort[1] = 0;
    if ((smem_u32(sm) & 1023u) != 0u) {
      atomicOr(x.err, kErrStreamBounds);
      *s_abort = 1;
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == 9) {
    tc5::tmem_alloc(smem_u32(s_tmem), kXmTmemCols);
    tc5::tmem_relinquish();
  }
  if (tid < kXmRows) s_tok[tid] = (float)(tid / x.G);
  // Columns of a step that hold no query (128 is not a multiple of G): no load writes their rows of the Q tiles, which
  // are zero from here on, and their log-sum-exp is +inf, so that they weigh nothing.
  {
    const int pad = kXmRows - tps * x.G;
    for (int i = tid; i < 2 * pad * 8; i += kXmThreads) {
      const int chunk = i & 7, r = tps * x.G + (i >> 3) % pad, half = (i >> 3) / pad;
      *reinterpret_cast<uint4*>(sm + 2 * kXmKBytes + half * (kXmQBytes / 2) + r * 128 + chunk * 16) = make_uint4(0u, 0u, 0u, 0u);
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
        v = e.ok && e.t > 0 ? (e.n + e.t + kXmItemKeys - 1) / kXmItemKeys : 0;
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
  // (a replayed graph's sequences may have outgrown the room for parts: every CTA sees the same)
  const int parts = s_item0[x.seqs.n] * p.plan.lh <= p.mass_items ? p.mass_parts : 1;
  const XmShared sh{s_n, s_item0, s_item0[x.seqs.n] * p.plan.lh * parts, parts};
  const int n_items = max(0, (sh.n_work - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x);
  auto slab_of = [&](const XmCursor& c) { return ((x.layer0 + c.layer) * x.Nb + x.seqs.b0 + c.s) * x.Hkv + c.h; };

  if (warp == 8) {
    // ================= the warp that loads Q, and K of 16-bit rows =================
    if (lane == 0 && *reinterpret_cast<volatile int*>(p.stop) != 0) *s_abort = 1;
    __syncwarp();
    XmCursor cur;
    cur.ord = 0;
    xm_seek(cur, 0, n_items, p, sh, true);
    int g = 0;
    while (cur.it < n_items && !*s_abort) {
      if constexpr (!KV8) {
        if (cur.ord > 0) mbar_wait(bar(6), (uint32_t)((cur.ord - 1) & 1), s_abort, x.err, p.wait_limit);  // the item before has read its K
        __syncwarp();
        if (!*s_abort && tc5::elect_one()) {
          const int slab = slab_of(cur);
          mbar_arrive_expect_tx(bar(0), 2 * kXmKBytes);
#pragma unroll
          for (int q = 0; q < 8; ++q)  // (boxes of 64 rows x 64 elements, as the attention's; those behind the slab's end come back as zeros)
            pf_tma_load(sK + (q >> 2) * kXmKBytes + ((q >> 1) & 1) * (kXmKBytes / 2) + (q & 1) * (kXmKBytes / 4), &tmK, 64 * ((q >> 1) & 1),
                        cur.k0 + kXmKeys * (q >> 2) + 64 * (q & 1), slab, bar(0));
        }
        __syncwarp();
      }
      for (int j = 0; j < cur.n_step; ++j, ++g) {
        if (g > 0) mbar_wait(bar(3), (uint32_t)((g - 1) & 1), s_abort, x.err, p.wait_limit);  // both groups' S of the step before have read its Q
        __syncwarp();
        if (*s_abort) break;
        if (tc5::elect_one()) {
          const uint32_t bb = bar(1);
          const int tok = cur.layer * x.total + x.seqs.tok0[cur.s] + (cur.lo + j) * tps;
          mbar_arrive_expect_tx(bb, 256u * (uint32_t)(x.G * tps));
          pf_tma_load(sQ, &tmQ, 0, cur.h * x.G, tok, bb);
          pf_tma_load(sQ + kXmQBytes / 2, &tmQ, 64, cur.h * x.G, tok, bb);
        }
        __syncwarp();
      }
      ++cur.ord;
      xm_seek(cur, cur.it + 1, n_items, p, sh, true);
    }
    if (*s_abort && lane == 0) {
      atomicOr(p.stop, 1);
      for (int i = KV8 ? 1 : 0; i < 2; ++i)
        for (uint32_t ph = 0; ph < 2; ++ph)
          for (uint32_t w = 0; w < (1u << 16); ++w)
            if (mbar_try_wait(bar(i), ph)) break;
    }
  } else if (warp == 9) {
    // ================= the warp that issues S = K Q^T, a group's after the other's =================
    constexpr uint32_t idesc = KV8 ? tc5::idesc_f16_f32(kXmKeys, kXmRows, 0, 0) : tc5::idesc_bf16_f32(kXmKeys, kXmRows, 0, 0);
    const uint64_t dK = tc5::smem_desc_sw128(sK, 16, 1024);
    const uint64_t dQ = tc5::smem_desc_sw128(sQ, 16, 1024);
    XmCursor cur;
    cur.ord = 0;
    xm_seek(cur, 0, n_items, p, sh, true);
    int g = 0;
    while (cur.it < n_items && !*s_abort) {
      mbar_wait(bar(0), (uint32_t)(cur.ord & 1), s_abort, x.err, p.wait_limit);
      for (int j = 0; j < cur.n_step; ++j, ++g) {
        mbar_wait(bar(1), (uint32_t)(g & 1), s_abort, x.err, p.wait_limit);
#pragma unroll
        for (int grp = 0; grp < 2; ++grp) {
          if (g > 0) mbar_wait(bar(4 + grp), (uint32_t)((g - 1) & 1), s_abort, x.err, p.wait_limit);
          __syncwarp();
          tc5::fence_after_sync();
          if (*s_abort) break;
          const uint64_t dKg = dK + (uint64_t)(grp * (kXmKBytes >> 4));
          if (tc5::elect_one()) {
#pragma unroll
            for (int kk = 0; kk < 8; ++kk)
              tc5::mma_bf16_ss(tmem + 128u * (uint32_t)grp, dKg + (uint64_t)((kk >> 2) * (kXmKBytes >> 5) + (kk & 3) * 2),
                               dQ + (uint64_t)((kk >> 2) * (kXmQBytes >> 5) + (kk & 3) * 2), idesc, kk > 0);
            tc5::mma_commit(bar(2 + grp));
            if (grp == 1 && j == cur.n_step - 1) tc5::mma_commit(bar(6));
          }
          __syncwarp();
        }
        if (*s_abort) break;
      }
      ++cur.ord;
      xm_seek(cur, cur.it + 1, n_items, p, sh, true);
    }
    if (*s_abort && tc5::elect_one()) {
      atomicOr(p.stop, 1);
      tc5::mma_commit(bar(7));
      for (uint32_t w = 0; w < kPfSpinLimit; ++w)
        if (mbar_try_wait(bar(7), 0u)) break;
    }
  } else {
    // ================= compute warps: thread = key = tensor-memory lane =================
    const int wg = warp >> 2, wq = warp & 3;
    const int row_in = wg * kXmKeys + wq * 32 + lane;
    const uint32_t t_row = tmem + 128u * (uint32_t)wg + ((uint32_t)(wq * 32) << 16);
    const uint32_t s_add = smem_u32(s_warp + warp * kXmWarpFloats);  // a column's negated log-sum-exp, less its part of the bias
    const uint32_t s_slope = s_add + 4 * kXmRows;                    // a column's negated slope
    const uint32_t s_token = smem_u32(s_tok), abort_flag = bar0 + 124u;
    XmCursor cur;
    cur.ord = 0;
    xm_seek(cur, 0, n_items, p, sh, false);
    int g = 0;
    while (cur.it < n_items) {
      const int j = cur.k0 + row_in;
      const bool mine = j < cur.n + cur.t;
      const size_t row = (size_t)slab_of(cur) * x.cap + j;
      const int prefix = x.seqs.prefix[cur.s], n_step = cur.n_step;
      if constexpr (KV8) {
        // 8-bit rows: this warp widens its own 32 rows, once the item before has read its K
        if (n_step > 0) {
          const uint8_t* src = static_cast<const uint8_t*>(x.K) + (size_t)slab_of(cur) * x.cap * 128;
          XtCodes codes[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) xt_load_codes(codes[q], src, cur.k0 + wg * kXmKeys + wq * 32 + 8 * q, cur.n + cur.t, lane);
          if (cur.ord > 0) xt_wait(bar(6), (uint32_t)((cur.ord - 1) & 1), abort_flag, p);
#pragma unroll
          for (int q = 0; q < 4; ++q) xt_store_codes<false>(codes[q], sm + wg * kXmKBytes, kXmKBytes / 2, wq * 32 + 8 * q, lane);
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(0));
        }
      }
      // the tokens that see row j: [i_lo, i_hi)
      int i_lo = j < cur.n + prefix ? 0 : j - cur.n, i_hi = mine ? cur.t : 0;
      float rel = 0.f;
      if constexpr (MODS) {
        const int at = mine ? x.pos[row] - x.held[kExtSeqs + cur.s] : 0;  // the row's position, the chunk's first token being 0
        rel = (float)at;
        if (x.window > 0) {
          i_lo = max(i_lo, (int)max(0ll, (long long)at - x.window + 1));  // (in 64 bits: a window may be as wide as an int)
          i_hi = (int)min((long long)i_hi, max(0ll, (long long)at + x.window));
        }
        if (x.slopes) {
          __syncwarp();
#pragma unroll
          for (int o = 0; o < kXmRows; o += 32) sts_f(s_slope + 4u * (uint32_t)(o + lane), x.slopes[cur.h * x.G + (o + lane) % x.G] * -1.4426950408889634f);
        }
      }
      const float* lse = x.lse + ext_lse_index(x, cur.layer, cur.h, x.seqs.tok0[cur.s]);
      const int all_rows = cur.t * x.G, step_rows = tps * x.G;
      auto ask = [&](int step, int off) {  // a step's negated log-sum-exp of column lane + off
        const int r = (cur.lo + step) * step_rows + lane + off;
        return lane + off < step_rows && r < all_rows ? -__ldcg(lse + r) : -CUDART_INF_F;
      };
      float la[kXmRows / 32];
#pragma unroll
      for (int o = 0; o < kXmRows / 32; ++o) la[o] = n_step > 0 ? ask(0, 32 * o) : 0.f;
      const bool biased = MODS && x.slopes != nullptr;
      float total = 0.f;
#pragma unroll 1
      for (int st = 0; st < n_step; ++st, ++g) {
        __syncwarp();
#pragma unroll
        for (int o = 0; o < kXmRows / 32; ++o) {
          const uint32_t at = 4u * (uint32_t)(32 * o + lane);
          sts_f(s_add + at, biased ? fmaf(lds_f(s_slope + at), lds_f(s_token + at), la[o]) : la[o]);
          if (st + 1 < n_step) la[o] = ask(st + 1, 32 * o);
        }
        __syncwarp();
        const int i0 = (cur.lo + st) * tps;
        const int rows = min(step_rows, all_rows - (cur.lo + st) * step_rows);
        const int c_lo = min(kXmRows, max(0, (i_lo - i0) * x.G)), c_hi = min(rows, max(0, (min(i_hi, i0 + tps) - i0) * x.G));
        const bool full = __all_sync(0xffffffffu, c_lo == 0 && c_hi == step_rows);
        const float off0 = (float)i0 - rel;
        const bool beside = biased && prefix > 0;  // rows of later positions may be seen
        xt_wait(bar(2 + wg), (uint32_t)(g & 1), abort_flag, p);
        tc5::fence_after_sync();
        uint64_t sum2[2] = {0ull, 0ull};
#pragma unroll 1
        for (int hb = 0; hb < rows; hb += 32) {
          uint32_t sv[32];
          tc5::tmem_ld32(t_row + (uint32_t)hb, sv);
          tc5::tmem_wait_ld();
          if (hb + 32 >= rows) {  // all has been read: S may be written again
            tc5::fence_before_sync();
            mbar_arrive(bar(4 + wg));
          }
          float scale = p.scale_log2;
          if constexpr (MODS) {
            if (x.cap_logit > 0.f) scale = xt_cap(sv, p);
          }
          const uint64_t scale2 = tc5::f2_pack(scale, scale), off2 = tc5::f2_pack(off0, off0);
          auto add_up = [&](auto masked) {
#pragma unroll
            for (int c = 0; c < 32; c += 4) {
              float4 add = lds_f4(s_add + 4u * (uint32_t)(hb + c));
              if constexpr (MODS) {
                // (the bias of column c: - slope_c (off0 + token_c); the token's part is in s_add)
                float4 ns = make_float4(0.f, 0.f, 0.f, 0.f);
                if (biased) ns = lds_f4(s_slope + 4u * (uint32_t)(hb + c));
                if (!biased) {
                } else if (beside) {
                  const float4 tk = lds_f4(s_token + 4u * (uint32_t)(hb + c));
                  add.x += ns.x * (fabsf(off0 + tk.x) - tk.x);
                  add.y += ns.y * (fabsf(off0 + tk.y) - tk.y);
                  add.z += ns.z * (fabsf(off0 + tk.z) - tk.z);
                  add.w += ns.w * (fabsf(off0 + tk.w) - tk.w);
                } else {
                  tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(ns.x, ns.y), off2, tc5::f2_pack(add.x, add.y)), add.x, add.y);
                  tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(ns.z, ns.w), off2, tc5::f2_pack(add.z, add.w)), add.z, add.w);
                }
              }
              float y[4];
              tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), scale2, tc5::f2_pack(add.x, add.y)), y[0], y[1]);
              tc5::f2_unpack(tc5::f2_fma(tc5::f2_pack(__uint_as_float(sv[c + 2]), __uint_as_float(sv[c + 3])), scale2, tc5::f2_pack(add.z, add.w)), y[2], y[3]);
              if constexpr (decltype(masked)::value) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                  if (hb + c + u < c_lo || hb + c + u >= c_hi) y[u] = -CUDART_INF_F;  // weight 0, whatever the logit is
              }
              sum2[0] = tc5::f2_add(sum2[0], tc5::f2_pack(fast_exp2(y[0]), fast_exp2(y[1])));
              sum2[1] = tc5::f2_add(sum2[1], tc5::f2_pack(fast_exp2(y[2]), fast_exp2(y[3])));
            }
          };
          if (full) add_up(std::false_type{});
          else add_up(std::true_type{});
        }
        float e, o;
        tc5::f2_unpack(tc5::f2_add(sum2[0], sum2[1]), e, o);
        total += e + o;
      }
      if (parts == 1) {
        if (mine && !*s_abort) ext_emit_mass(x, row, total);
      } else {
        // a part: left in the scratch; the last to finish adds them in order
        float* part = p.mass_part + (size_t)cur.item * parts * kXmItemKeys + row_in;
        __stcg(part + cur.part * kXmItemKeys, total);
        __threadfence();
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (tid == 0) *s_flag = atomicAdd(p.mass_counters + cur.item, 1u) == (unsigned)(parts - 1);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const bool last = *s_flag != 0;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (last) {
          __threadfence();
          float sum = 0.f;
#pragma unroll 4
          for (int k = 0; k < parts; ++k) sum += __ldcg(part + k * kXmItemKeys);
          if (mine && !*s_abort) ext_emit_mass(x, row, sum);
        }
      }
      if (n_step > 0) ++cur.ord;
      xm_seek(cur, cur.it + 1, n_items, p, sh, false);
    }
  }
  tc5::fence_before_sync();
  __syncthreads();
  if (warp == 9) tc5::tmem_dealloc(tmem, kXmTmemCols);
}

}  // namespace dynts
