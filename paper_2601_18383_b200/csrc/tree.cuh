// Trees of drafted tokens.  A chunk's nodes name their parents (a node before it in the chunk, or -1); node i attends to
// the rows held, to its ancestors and to itself.
//
// tree_plan_kernel numbers the nodes in preorder: order_i = its place in a walk that visits a node before its
// children (siblings in the order of the chunk), size_i = nodes of its subtree.  Then
//     j is i or an ancestor of i   <=>   0 <= order_i - order_j < size_j,
// one subtraction and one comparison for each (query, row), where a mask of bits would take a word per 32 rows of the
// chunk and query.  depth_i gives the positions.  Sizes, depths and the sums along a path come by pointer doubling: after k
// rounds a node knows the 2^k nearest ancestors' part, so a tree takes log2(depth) rounds whatever its shape.
// One CTA per sequence, a thread per node: bound by the latency of a launch and of about ten barriers (2 us).
//
// tree_accept_kernel walks down from node 0 while a child's drafted token is the token drawn at the node.
// tree_move_kernel brings an accepted path's rows together behind the rows held.
#pragma once

#include "common.cuh"
#include "extend.cuh"

namespace dynts {

constexpr int kTreeNodes = 1024;  // of a sequence's tree
constexpr int kErrTree = 32;      // device status bit: a parent not before its child, or a path out of order

struct TreeSeqs {
  int n, b0;
  int tok0[kExtSeqs + 1];
};

__global__ void __launch_bounds__(kTreeNodes) tree_plan_kernel(const __grid_constant__ TreeSeqs q, const int* parents, const int* tot, int4* tree, int* positions, int* err) {
  __shared__ int s_up[kTreeNodes], s_a[kTreeNodes], s_b[kTreeNodes];
  const int s = blockIdx.x, i = threadIdx.x, t0 = q.tok0[s], t = q.tok0[s + 1] - t0;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int parent = -1;
  if (i < t) {
    parent = parents[t0 + i];
    if (parent < -1 || parent >= i) {
      atomicOr(err, kErrTree);
      parent = -1;
    }
  }
  // subtree sizes and depths: up = the ancestor 2^k above, size = nodes less than 2^k below, depth = steps up to there
  int up = parent, size = 1, depth = parent >= 0 ? 1 : 0;
  while (true) {
    s_up[i] = up;
    s_a[i] = size;
    s_b[i] = depth;
    if (!__syncthreads_or(up >= 0)) break;
    const int up2 = up >= 0 ? s_up[up] : -1, more = up >= 0 ? s_b[up] : 0;
    __syncthreads();
    if (up >= 0) atomicAdd(&s_a[up], size);  // (whole numbers: any order)
    __syncthreads();
    size = s_a[i];
    depth += more;
    up = up2;
    __syncthreads();
  }
  // what precedes a node among its siblings, summed along its path
  s_up[i] = parent;
  s_a[i] = size;
  __syncthreads();
  int before = 0;
  for (int y = max(parent, 0); y < i && i < t; ++y)
    if (s_up[y] == parent) before += s_a[y];
  up = parent;
  int order = before;
  __syncthreads();
  while (true) {
    s_up[i] = up;
    s_b[i] = order;
    if (!__syncthreads_or(up >= 0)) break;
    const int up2 = up >= 0 ? s_up[up] : -1, more = up >= 0 ? s_b[up] : 0;
    __syncthreads();
    order += more;
    up = up2;
  }
  if (i < t) {
    tree[t0 + i] = make_int4(order + depth, size, depth, parent);
    if (positions) positions[t0 + i] = tot[q.b0 + s] + depth;
  }
}

// A warp per sequence: children of the node reached are looked for 32 nodes at a time, the lowest index wins.
__global__ void __launch_bounds__(128) tree_accept_kernel(const __grid_constant__ TreeSeqs q, const int* parents, const int* drafted, const int* drawn, int* path, int max_path,
                                                          int* accepted, int* next) {
  const int s = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x & 31;
  if (s >= q.n) return;
  const int t0 = q.tok0[s], t = q.tok0[s + 1] - t0, b = q.b0 + s;
  int count = 0, at = t > 0 ? 0 : -1, token = -1;
  while (at >= 0) {
    if (lane == 0) path[(size_t)b * max_path + count] = at;
    ++count;
    token = drawn[t0 + at];
    int child = -1;
    if (count < max_path && token >= 0)
      for (int j = at + 1; j < t && child < 0; j += 32) {
        const unsigned hit = __ballot_sync(0xffffffffu, j + lane < t && parents[t0 + j + lane] == at && drafted[t0 + j + lane] == token);
        if (hit) child = j + __ffs(hit) - 1;
      }
    at = child;
  }
  for (int k = count + lane; k < max_path; k += 32) path[(size_t)b * max_path + k] = -1;
  if (lane == 0) {
    accepted[b] = count;
    next[b] = token;
  }
}

struct TreeMoveParams {
  TreeSeqs seqs;      // tok0: running sums of the rows accepted
  int staged[kExtSeqs];
  const int* path;    // [Nb][path_stride]
  long long path_stride;
  uint8_t* K;
  uint8_t* V;
  int* pos;
  float* score;
  float* comp;
  int* len;
  int* tot;
  int* active;
  int* err;
  int Nb, Hkv, cap, row_bytes;
};

// The rows of a path are in order and lie among the staged ones.
__device__ __forceinline__ bool tree_path_ok(const TreeMoveParams& p, const int* path, int count, int staged, int n) {
  bool ok = n >= 0 && n + staged <= p.cap;
  for (int k = (int)threadIdx.x; k < count; k += (int)blockDim.x) ok = ok && path[k] >= 0 && path[k] < staged && (k == 0 || path[k - 1] < path[k]);
  return __syncthreads_and(ok);
}

// Rows n + path[k] -> n + k of one slab: sources and targets both ascend and no source lies before its target, so blocks of
// pieces, each read whole before it is written, overwrite nothing unread.  Grid: x over (layer, KV head), y over sequences.
__global__ void __launch_bounds__(256) tree_move_kernel(const __grid_constant__ TreeMoveParams p) {
  const int s = blockIdx.y, b = p.seqs.b0 + s, count = p.seqs.tok0[s + 1] - p.seqs.tok0[s];
  if (count == 0) return;
  const int* path = p.path + (size_t)b * p.path_stride;
  const int n = p.len[b], layer = blockIdx.x / p.Hkv, h = blockIdx.x - layer * p.Hkv;
  if (!tree_path_ok(p, path, count, p.staged[s], n)) return;
  const size_t row0 = (((size_t)layer * p.Nb + b) * p.Hkv + h) * p.cap + n;
  const int pieces = p.row_bytes / 16, all = count * 2 * pieces;
  for (int w0 = 0; w0 < all; w0 += (int)blockDim.x) {
    const int w = w0 + (int)threadIdx.x, k = w / (2 * pieces), c = w - k * 2 * pieces;
    uint8_t* base = c < pieces ? p.K : p.V;
    const size_t at = (size_t)(c < pieces ? c : c - pieces) * 16;
    uint4 x = make_uint4(0u, 0u, 0u, 0u);
    if (w < all) x = *reinterpret_cast<const uint4*>(base + (row0 + path[k]) * p.row_bytes + at);
    __syncthreads();
    if (w < all) *reinterpret_cast<uint4*>(base + (row0 + k) * p.row_bytes + at) = x;
    __syncthreads();
  }
  const int tot = p.tot[b];
  for (int k0 = 0; k0 < count; k0 += (int)blockDim.x) {
    const int k = k0 + (int)threadIdx.x;
    const float sc = k < count ? p.score[row0 + path[k]] : 0.f;
    __syncthreads();
    if (k < count) {
      p.score[row0 + k] = sc;
      p.comp[row0 + k] = 0.f;
      p.pos[row0 + k] = tot + k;
    }
    __syncthreads();
  }
}

// Behind it: the lengths, of the sequences whose path was in order.  A CTA per sequence.
__global__ void __launch_bounds__(128) tree_lengths_kernel(const __grid_constant__ TreeMoveParams p) {
  const int s = blockIdx.x, b = p.seqs.b0 + s, count = p.seqs.tok0[s + 1] - p.seqs.tok0[s];
  if (count == 0) return;
  const bool ok = tree_path_ok(p, p.path + (size_t)b * p.path_stride, count, p.staged[s], p.len[b]);
  if (threadIdx.x != 0) return;
  if (!ok) {
    atomicOr(p.err, kErrTree);
    return;
  }
  p.len[b] += count;
  p.tot[b] += count;
  p.active[b] = 1;
}

}  // namespace dynts
