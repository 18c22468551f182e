// Shared by the kernels of speculative decoding (draft*.cu): arguments, the tree of drafts, where a node's tensors lie.
#pragma once

#include "rattn_internal.h"

namespace rattn {
namespace draft {

constexpr int kMaxNodes = RATTN_DRAFT_MAX_NODES;

struct DraftArgs {
  const void* q; const void* k; const void* v; void* out;
  const int* parents;
  void* k_ring; void* v_ring; float* state;
  const float* gamma_swa; const float* gamma_rla;
  const int* pos_dev; const int* path; const int* n_accepted;
  int B, H_q, H_kv, N, d, w, group, dtype, phi, layout, pos;
  unsigned flags;
  float scale, eps;
};

// Element offset of node n of head h (of H) of batch entry b in a tensor of nodes.
__device__ __forceinline__ size_t node_at(const DraftArgs& a, int b, int h, int H, int n) {
  return (a.layout == RATTN_LAYOUT_BHTD ? ((size_t)b * H + h) * a.N + n : ((size_t)b * a.N + n) * H + h) * a.d;
}
__device__ __forceinline__ int entry_pos(const DraftArgs& a, int b) { return a.pos_dev ? max(a.pos_dev[b], 0) : a.pos; }

// Ring slots by age.  The slot that position pos would take is pos % w; slot s holds token pos - w + rank(s), which exists
// for rank >= w - min(pos, w).  A node at depth e sees the slots of rank >= e in its window and those below through the
// linear branch.
struct RingAge {
  int w, head, first;            // head: pos % w; first: lowest rank that holds a token
  __device__ __forceinline__ RingAge(int pos, int w_) : w(w_), head(pos % w_), first(pos < w_ ? w_ - pos : 0) {}
  __device__ __forceinline__ int rank(int slot) const { return slot >= head ? slot - head : slot - head + w; }
  __device__ __forceinline__ int slot(int rank) const { return rank + head >= w ? rank + head - w : rank + head; }
};

// Depth of node i, or -1 where it is no part of the tree.  par: the entry's parents in shared memory.  Chains of parents
// fall strictly, so the walk ends.
__device__ __forceinline__ int node_depth(const int* par, int i) {
  int e = 0;
  for (;;) {
    const int p = par[i];
    if (p == -1) return e;
    if (p < 0 || p >= i) return -1;
    i = p;
    ++e;
  }
}

// One bit per node: the node itself and its ancestors.
struct NodeSet { uint32_t w[kMaxNodes / 32]; };
__device__ __forceinline__ void node_path(const int* par, int i, NodeSet* s) {
#pragma unroll
  for (int j = 0; j < kMaxNodes / 32; ++j) s->w[j] = 0u;
  for (;;) {
#pragma unroll
    for (int j = 0; j < kMaxNodes / 32; ++j) s->w[j] |= (i >> 5) == j ? 1u << (i & 31) : 0u;
    const int p = par[i];
    if (p < 0 || p >= i) return;
    i = p;
  }
}

__device__ __forceinline__ float wmax(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float wsum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

// 1 / sqrt(mean(x^2) + eps) of a row of 32 C values, C of them in each lane.  Squares are summed in fp32, which ends at values of
// some 1e18: a row whose sum overflows is summed again from values scaled down by kDown, eps likewise.
constexpr float kDown = 0x1p-100f;
template <int C>
__device__ __forceinline__ float row_inv_rms(const float (&x)[C], float eps) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i) s += x[i] * x[i];
  s = wsum(s);
  if (s != INFINITY) return rsqrtf(s / (32 * C) + eps);
  s = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i) s += (x[i] * kDown) * (x[i] * kDown);
  return rsqrtf(wsum(s) / (32 * C) + eps * kDown * kDown) * kDown;
}

// How many clusters of `cluster` CTAs (2, 4 or 8) of the kernel run at once on the current device, asked of the driver once per
// device.  Fewer than its SMs have room for: a cluster lies within one GPC, and what is left of a GPC takes none.
template <auto Kernel>
cudaError_t clusters_at_once(int cluster, int threads, int smem, int* n) {
  static std::atomic<int> known[kMaxDevices][4];             // 1 more than the answer
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::atomic<int>& slot = known[dev][cluster >> 2 ? (cluster >> 3) + 2 : 1];
  if (const int k = slot.load(std::memory_order_relaxed)) {
    *n = k - 1;
    return cudaSuccess;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)cluster);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = (size_t)smem;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  e = cudaOccupancyMaxActiveClusters(n, Kernel, &cfg);
  if (e == cudaSuccess) slot.store(*n + 1, std::memory_order_relaxed);
  return e;
}

cudaError_t launch_generic(const DraftArgs& a, cudaStream_t s);
cudaError_t launch_commit(const DraftArgs& a, cudaStream_t s);
// The tensor-core kernel and its status word (RATTN_ERR_TIMEOUT once a bounded wait has expired; reading clears it).
bool tc_applies(const DraftArgs& a);
cudaError_t launch_tc(const DraftArgs& a, cudaStream_t s);
int tc_status(cudaStream_t s, cudaError_t* err);

}  // namespace draft
}  // namespace rattn
