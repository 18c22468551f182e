// Entry of the accepted tokens into ring and state (rattn_draft_commit): what n single-token steps would leave,
//
//   S += sum_a phi(k_old(a))^T v_old(a),     ring slot (pos + a) % w = token a,        a = 0 .. n-1,
//
// old(a) = token pos + a - w: a ring slot's for a < w, an accepted token's behind that.  One read and one write of the
// state (64 KB each at d = 128) is nearly all of the traffic, so HBM bounds it, or latency for few heads: a CTA has its share
// of the state's rows in registers, requested before anything else, and the ring rows that the first eight tokens would push
// out are requested before it is known how many tokens there are.  Few heads of d = 128 are shared by clusters of four CTAs.
// Tokens are added in order, as single steps would (fp32).
//
// The slots that the new tokens take are those that the old ones leave: the CTAs of a head meet at a barrier between the last
// read of an old token and the first write of a new one.
#include "draft_internal.h"

namespace rattn {
namespace draft {
namespace {

constexpr int DC_THREADS = 256, DC_TOKENS = DC_THREADS / 32;        // tokens whose phi(k), v lie in shared memory at a time

template <typename T, int D, int CS>
__global__ void __launch_bounds__(DC_THREADS, CS == 1 ? 2 : 4) draft_commit_kernel(const __grid_constant__ DraftArgs a) {
  constexpr int C = D / 32, CG = D / 4, LANES = DC_THREADS / CG, ROWS = D / CS / LANES;
  __shared__ __align__(16) float fk[DC_TOKENS][D];
  __shared__ __align__(16) float vo[DC_TOKENS][D];
  __shared__ int path[kMaxNodes];
  __shared__ int n_s;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, w = a.w;
  const int z = blockIdx.x / CS, rank = blockIdx.x % CS, b = z / a.H_kv, hk = z % a.H_kv;
  const int c4 = (tid % CG) * 4, row0 = rank * (D / CS) + tid / CG;
  if (tid == 0) n_s = a.N;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");        // the inputs may come from the kernel before
  const int pos = entry_pos(a, b), n_raw = a.n_accepted[b];
  const int node = tid < a.N ? a.path[(size_t)b * a.N + tid] : -1;
  float* S = a.state + (size_t)z * D * D;
  float4 acc[ROWS];
#pragma unroll
  for (int i = 0; i < ROWS; ++i) acc[i] = *reinterpret_cast<const float4*>(S + (size_t)(row0 + i * LANES) * D + c4);
  T* kr = static_cast<T*>(a.k_ring) + (size_t)z * w * D;
  T* vr = static_cast<T*>(a.v_ring) + (size_t)z * w * D;
  const T* kn = static_cast<const T*>(a.k);
  const T* vn = static_cast<const T*>(a.v);
  const int head = pos % w, a0 = pos < w ? w - pos : 0;     // a0: the first accepted token that pushes one out
  // this warp's token of the first eight, where it is one of the ring
  T k1[C], v1[C];
  const int at1 = a0 + warp;
  if (at1 < a.N && at1 < w) {
    const size_t from = (size_t)((head + at1) % w) * D + lane;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      k1[i] = kr[from + 32 * i];
      v1[i] = vr[from + 32 * i];
    }
  }
  __syncthreads();
  if (tid < a.N) {
    path[tid] = node;
    if (node < 0 || node >= a.N) atomicMin(&n_s, tid);
  }
  __syncthreads();
  const int n = min(n_s, max(n_raw, 0));
  if (n == 0) return;                                       // the same for the whole cluster

  for (int t0 = a0; t0 < n; t0 += DC_TOKENS) {
    const int m = min(DC_TOKENS, n - t0), at = t0 + warp;
    if (warp < m) {
      if (t0 != a0 || at >= w) {
        const bool ring = at < w;
        const size_t from = ring ? (size_t)((head + at) % w) * D : node_at(a, b, hk, a.H_kv, path[at - w]);
#pragma unroll
        for (int i = 0; i < C; ++i) {
          k1[i] = ((ring ? kr : kn) + from)[lane + 32 * i];
          v1[i] = ((ring ? vr : vn) + from)[lane + 32 * i];
        }
      }
      float x[C];
#pragma unroll
      for (int i = 0; i < C; ++i) {
        x[i] = (float)k1[i];
        vo[warp][lane + 32 * i] = (float)v1[i];
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
      for (int i = 0; i < C; ++i) fk[warp][lane + 32 * i] = x[i];
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
  if (CS > 1) {                                             // every old token has been read
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  constexpr int V16 = D * (int)sizeof(T) / 16;              // 16-byte pieces of a row
  const int first = n > w ? n - w : 0;                      // earlier ones have been pushed out by the path itself
  for (int i = tid; i < (n - first) * 2 * V16; i += DC_THREADS) {
    const int t = first + i / (2 * V16), piece = i % V16;
    if (t % CS != rank) continue;
    const bool is_v = (i / V16) & 1;
    const size_t from = node_at(a, b, hk, a.H_kv, path[t]), to = (size_t)((head + (t % w)) % w) * D;
    reinterpret_cast<uint4*>((is_v ? vr : kr) + to)[piece] = reinterpret_cast<const uint4*>((is_v ? vn : kn) + from)[piece];
  }
}

template <typename T, int D, int CS>
cudaError_t launch_commit_cs(const DraftArgs& a, cudaStream_t s) {
  KernelTimer kt("draft_commit", s);
  const cudaError_t e = launch_pdl_cluster(draft_commit_kernel<T, D, CS>, dim3((unsigned)(a.B * a.H_kv * CS)), dim3(DC_THREADS), 0, s,
                                           true, CS, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return cudaGetLastError();
}

// d = 128: a head to a cluster of four CTAs while all of these run at once, to one CTA beyond; d = 64, with a quarter of the
// state: one CTA.  One CTA / four, bf16, states from HBM: d = 128, 8 heads 3.7 / 3.5 us, 64 6.6 / 5.9, 128 7.6 / 7.0, 148 6.7 / 9.8,
// 512 16.8 / 21.7 (the state's 67 MB at 4.1 TB/s; 1600 heads: 5.3); d = 64, 8 heads 2.4 / 2.8, 128 4.1 / 4.6, 512 8.1 / 15.7.
template <typename T, int D>
cudaError_t launch_commit_as(const DraftArgs& a, cudaStream_t s) {
  if constexpr (D == 128) {
    int n = 0;
    const cudaError_t e = clusters_at_once<draft_commit_kernel<T, D, 4>>(4, DC_THREADS, 0, &n);
    if (e != cudaSuccess) return e;
    if (a.B * a.H_kv <= n) return launch_commit_cs<T, D, 4>(a, s);
  }
  return launch_commit_cs<T, D, 1>(a, s);
}

}  // namespace

cudaError_t launch_commit(const DraftArgs& a, cudaStream_t s) {
  if (a.dtype == RATTN_BF16)
    return a.d == 128 ? launch_commit_as<__nv_bfloat16, 128>(a, s) : launch_commit_as<__nv_bfloat16, 64>(a, s);
  return a.d == 128 ? launch_commit_as<float, 128>(a, s) : launch_commit_as<float, 64>(a, s);
}

}  // namespace draft
}  // namespace rattn
