// Entry of the accepted tokens into ring and state (rattn_draft_commit): what n single-token steps would leave,
//
//   S += sum_a phi(k_old(a))^T v_old(a),     ring slot (pos + a) % w = token a,        a = 0 .. n-1,
//
// old(a) = token pos + a - w: a ring slot's for a < w, an accepted token's behind that.  One read and one write of the
// state (64 KB each at d = 128) is nearly all of the traffic, so HBM bounds it, or latency for few heads: a (batch entry, K/V
// head) is shared by a cluster of CTAs, each with a share of the state's rows in registers, requested before anything else.
// Tokens are added in order, as single steps would (fp32).
//
// The slots that the new tokens take are those that the old ones leave: the cluster meets at a barrier between the last
// read of an old token and the first write of a new one.
#include "draft_internal.h"

namespace rattn {
namespace draft {
namespace {

constexpr int DC_THREADS = 256, DC_CLUSTER = 4, DC_TOKENS = 16;     // tokens whose phi(k), v lie in shared memory at a time

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

template <typename T, int D>
__global__ void __launch_bounds__(DC_THREADS) draft_commit_kernel(const __grid_constant__ DraftArgs a) {
  constexpr int C = D / 32, CG = D / 4, LANES = DC_THREADS / CG, ROWS = D / DC_CLUSTER / LANES;
  __shared__ __align__(16) float fk[DC_TOKENS][D];
  __shared__ __align__(16) float vo[DC_TOKENS][D];
  __shared__ int path[kMaxNodes];
  __shared__ int n_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int z = blockIdx.x / DC_CLUSTER, rank = blockIdx.x % DC_CLUSTER, b = z / a.H_kv, hk = z % a.H_kv;
  const int c4 = (tid % CG) * 4, row0 = rank * (D / DC_CLUSTER) + tid / CG;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");        // the inputs may come from the kernel before
  float* S = a.state + (size_t)z * D * D;
  float4 acc[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) acc[i] = *reinterpret_cast<const float4*>(S + (size_t)(row0 + i * LANES) * D + c4);
  if (tid == 0) n_s = min(max(a.n_accepted[b], 0), a.N);
  __syncthreads();
  if (tid < a.N) {
    path[tid] = a.path[(size_t)b * a.N + tid];
    if (path[tid] < 0 || path[tid] >= a.N) atomicMin(&n_s, tid);
  }
  __syncthreads();
  const int n = n_s, w = a.w, pos = entry_pos(a, b), head = pos % w;
  if (n == 0) return;                                       // the same for the whole cluster
  T* kr = static_cast<T*>(a.k_ring) + (size_t)z * w * D;
  T* vr = static_cast<T*>(a.v_ring) + (size_t)z * w * D;
  const T* kn = static_cast<const T*>(a.k);
  const T* vn = static_cast<const T*>(a.v);

  const int a0 = pos < w ? w - pos : 0;                     // the first accepted token that pushes one out
  for (int t0 = a0; t0 < n; t0 += DC_TOKENS) {
    const int m = min(DC_TOKENS, n - t0);
    for (int t = warp; t < m; t += DC_THREADS / 32) {
      const int at = t0 + t;
      const size_t from = at < w ? (size_t)((head + at) % w) * D : node_at(a, b, hk, a.H_kv, path[at - w]);
      const T* ko = (at < w ? kr : kn) + from;
      const T* vv = (at < w ? vr : vn) + from;
      float x[C];
#pragma unroll
      for (int i = 0; i < C; ++i) {
        x[i] = (float)ko[lane + 32 * i];
        vo[t][lane + 32 * i] = (float)vv[lane + 32 * i];
      }
      if (a.phi == RATTN_PHI_SOFTMAX) {
        float mx = x[0], s = 0.f;
#pragma unroll
        for (int i = 1; i < C; ++i) mx = fmaxf(mx, x[i]);
        mx = wmax(mx);
#pragma unroll
        for (int i = 0; i < C; ++i) s += x[i] = expf(x[i] - mx);
        const float inv = 1.f / wsum(s);
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] *= inv;
      } else if (a.phi == RATTN_PHI_RELU) {
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = fmaxf(x[i], 0.f);
      }
#pragma unroll
      for (int i = 0; i < C; ++i) fk[t][lane + 32 * i] = x[i];
    }
    __syncthreads();
    for (int t = 0; t < m; ++t) {
      const float4 v = *reinterpret_cast<const float4*>(&vo[t][c4]);
#pragma unroll
      for (int i = 0; i < ROWS; ++i) {
        const float f = fk[t][row0 + i * LANES];
        acc[i].x += f * v.x; acc[i].y += f * v.y; acc[i].z += f * v.z; acc[i].w += f * v.w;
      }
    }
    __syncthreads();
  }
  if (a0 < n) {
#pragma unroll
    for (int i = 0; i < ROWS; ++i) *reinterpret_cast<float4*>(S + (size_t)(row0 + i * LANES) * D + c4) = acc[i];
  }
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");    // every old token has been read
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  constexpr int V16 = D * (int)sizeof(T) / 16;              // 16-byte pieces of a row
  const int first = n > w ? n - w : 0;                      // earlier ones have been pushed out by the path itself
  for (int i = tid; i < (n - first) * 2 * V16; i += DC_THREADS) {
    const int t = first + i / (2 * V16), piece = i % V16;
    if (t % DC_CLUSTER != rank) continue;
    const bool is_v = (i / V16) & 1;
    const size_t from = node_at(a, b, hk, a.H_kv, path[t]), to = (size_t)((head + (t % w)) % w) * D;
    reinterpret_cast<uint4*>((is_v ? vr : kr) + to)[piece] = reinterpret_cast<const uint4*>((is_v ? vn : kn) + from)[piece];
  }
}

template <typename T, int D>
cudaError_t launch_commit_as(const DraftArgs& a, cudaStream_t s) {
  KernelTimer kt("draft_commit", s);
  const cudaError_t e = launch_pdl_cluster(draft_commit_kernel<T, D>, dim3((unsigned)(a.B * a.H_kv * DC_CLUSTER)), dim3(DC_THREADS),
                                           0, s, true, DC_CLUSTER, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_commit(const DraftArgs& a, cudaStream_t s) {
  if (a.dtype == RATTN_BF16)
    return a.d == 128 ? launch_commit_as<__nv_bfloat16, 128>(a, s) : launch_commit_as<__nv_bfloat16, 64>(a, s);
  return a.d == 128 ? launch_commit_as<float, 128>(a, s) : launch_commit_as<float, 64>(a, s);
}

}  // namespace draft
}  // namespace rattn
