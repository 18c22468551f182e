// Verification of drafted tokens (rattn_draft_verify): the walk down the tree and the token drawn behind it.
//
// With c the node accepted last and r, Z what the rejections under c have left of its row p (r = p, Z = 1 at first), node i under
// c is accepted if u q(x) Z < r(x); a rejection makes r' = max(r - Z q, 0), Z' = sum r'.  A test needs r at one token only, so
// the probabilities of all nodes' tokens under their parents are fetched at once, before the walk, and a rejection's sum
// Z' -- a pass over the vocabulary -- is formed only if another node under c is tested, or at the end, where the same
// pass serves the draw.  A chain that is accepted up to one rejection costs one pass over one row of p and q: that row is
// the traffic, and HBM bounds large batches, latency small ones.
//
// A batch entry has a cluster of CTAs; each takes a run of the vocabulary, each of its warps a run of that.  All threads of the
// cluster walk the tree alike (from shared memory; the sums are added in an order fixed by the sizes), so
// nothing but the partial sums passes between them, through distributed shared memory.  r is never stored: it is formed
// again from p, q and the list of Z.  Sums, r and comparisons are fp64: the drawn token is an index, and in fp32 the
// running sum over 10^5 tokens of 10^-5 would be off by as much as their probabilities.
#include "draft_internal.h"

namespace rattn {
namespace draft {
namespace {

constexpr int DV_THREADS = 512, DV_WARPS = DV_THREADS / 32, DV_CLUSTER = 8;

struct VerifyArgs {
  const int* tokens; const int* parents;
  const void* p; const void* q;
  const float* u;
  int* path; int* n_accepted; int* token;
  int B, N, V;
};

template <typename T> __device__ __forceinline__ float prob(T x) {      // negative and NaN count as 0
  const float f = (float)x;
  return f > 0.f ? f : 0.f;
}

__device__ __forceinline__ double wsum(double x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ double ld_cluster(const double* p, int rank) {
  uint32_t a;
  double v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
  asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(a) : "memory");
  return v;
}

// What the rejections under the current node have left of its row.
struct Left {
  int n;                         // rejections that count
  double Z[kMaxNodes];           // with a drafter's row: Z ahead of each of them
  int x[kMaxNodes];              // without: the token that each of them took out
};

template <typename T, bool DRAFT>
__device__ __forceinline__ double left_of(double p, double q, int x, const Left& l) {
  if (DRAFT) {
    for (int i = 0; i < l.n; ++i) p = fmax(p - l.Z[i] * q, 0.0);
  } else {
    for (int i = 0; i < l.n; ++i)
      if (l.x[i] == x) p = 0.0;
  }
  return p;
}

template <typename T, bool DRAFT>
__global__ void __launch_bounds__(DV_THREADS) draft_verify_kernel(const __grid_constant__ VerifyArgs a) {
  __shared__ int par[kMaxNodes], tok[kMaxNodes], path[kMaxNodes];
  __shared__ float u_s[kMaxNodes];
  __shared__ double pt[kMaxNodes], qt[kMaxNodes];
  __shared__ Left left;
  __shared__ double warp_sum[DV_WARPS];
  __shared__ double cta_sum[2];                             // in turns, so that a sum is not overwritten while others read it
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int b = blockIdx.x / DV_CLUSTER, rank = blockIdx.x % DV_CLUSTER, N = a.N, V = a.V;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");        // the inputs may come from the kernel before
  const T* p_rows = static_cast<const T*>(a.p) + (size_t)b * N * V;
  const T* q_rows = static_cast<const T*>(a.q) + (size_t)b * N * V;
  if (tid < N) {
    const int up = a.parents[(size_t)b * N + tid], x = a.tokens[(size_t)b * N + tid];
    par[tid] = up;
    tok[tid] = x;
    u_s[tid] = a.u[(size_t)b * N + tid];
    const bool real = up >= 0 && up < tid && x >= 0 && x < V;
    pt[tid] = real ? (double)prob(p_rows[(size_t)up * V + x]) : 0.0;
    qt[tid] = DRAFT ? (real ? (double)prob(q_rows[(size_t)up * V + x]) : 0.0) : 1.0;
  }
  if (tid == 0) left.n = 0;
  __syncthreads();

  const bool idle = par[0] != -1;
  if (idle) {                                               // the same for the whole cluster
    if (rank == 0) {
      if (tid < N) a.path[(size_t)b * N + tid] = -1;
      if (tid == 0) {
        a.n_accepted[b] = 0;
        a.token[b] = -1;
      }
    }
    return;
  }
  // runs of the vocabulary: this CTA's, this warp's
  const int per_cta = (V + DV_CLUSTER - 1) / DV_CLUSTER, per_warp = (per_cta + DV_WARPS - 1) / DV_WARPS;
  const int cta0 = min(rank * per_cta, V), cta1 = min(cta0 + per_cta, V);
  const int w0 = min(cta0 + warp * per_warp, cta1), w1 = min(w0 + per_warp, cta1);
  int turn = 0;
  // Sum of r over the vocabulary, with a rejection at Z that is not in the list yet (draft rows; pending).  Leaves the
  // warps' sums in warp_sum and the CTAs' in cta_sum[turn - 1].
  auto total = [&](int c, bool pending, double Z) -> double {
    const T* p = p_rows + (size_t)c * V;
    const T* q = q_rows + (size_t)c * V;
    double s = 0.0;
#pragma unroll 4
    for (int x = w0 + lane; x < w1; x += 32) {
      const double qx = DRAFT ? (double)prob(q[x]) : 0.0;
      double r = left_of<T, DRAFT>((double)prob(p[x]), qx, x, left);
      if (DRAFT && pending) r = fmax(r - Z * qx, 0.0);
      s += r;
    }
    s = wsum(s);
    if (lane == 0) warp_sum[warp] = s;
    __syncthreads();
    if (tid == 0) {
      double t = 0.0;
      for (int i = 0; i < DV_WARPS; ++i) t += warp_sum[i];
      cta_sum[turn & 1] = t;
    }
    cluster_sync();
    double t = 0.0;
    for (int r = 0; r < DV_CLUSTER; ++r) t += ld_cluster(&cta_sum[turn & 1], r);
    ++turn;
    return t;
  };

  constexpr double kTiny = 1.0 / (double)(1ull << 40);
  int c = 0, n = 1;
  double Z = 1.0, sum = 0.0;
  bool pending = false, summed = false;                     // summed: the last pass was over r as it is now
  // a rejection whose sum has not been formed
  auto settle = [&]() {
    const double s = total(c, true, Z);
    const bool counts = s > kTiny * Z;
    if (counts) {
      __syncthreads();
      if (tid == 0) left.Z[left.n++] = Z;
      __syncthreads();
      Z = s;
    }
    pending = false;
    summed = counts;
    sum = s;
  };
  if (tid == 0) path[0] = 0;
  for (int i = 1; i < N; ++i) {
    if (par[i] != c) continue;
    const int x = tok[i];
    if (x < 0 || x >= V) continue;
    if (pending) settle();
    const double r = left_of<T, DRAFT>(pt[i], qt[i], x, left);
    if ((double)u_s[i] * qt[i] * Z < r) {
      c = i;
      Z = 1.0;
      __syncthreads();
      if (tid == 0) {
        left.n = 0;
        path[n] = i;
      }
      __syncthreads();
      ++n;
      summed = false;
    } else if (DRAFT) {
      pending = true;
    } else {
      __syncthreads();
      if (tid == 0) left.x[left.n++] = x;
      __syncthreads();
      Z -= r;
    }
  }
  if (DRAFT && pending) settle();
  if (!summed) sum = total(c, false, 0.0);
  if (!(sum > 0.0) && left.n > 0) {                         // nothing left: the row as it is given
    __syncthreads();
    if (tid == 0) left.n = 0;
    __syncthreads();
    sum = total(c, false, 0.0);
  }
  // the draw: the CTA, the warp and the token in whose share the target lies
  if (!(sum > 0.0)) {
    if (rank == 0 && tid == 0) a.token[b] = -1;
  } else {
    const double target = (double)u_s[0] * sum;
    double run = 0.0, ahead = 0.0;                          // ahead: the sum in front of the owner's share
    int owner = -1, last = 0;
    for (int r = 0; r < DV_CLUSTER; ++r) {
      const double s = ld_cluster(&cta_sum[(turn - 1) & 1], r);
      if (s > 0.0) last = r;
      if (owner < 0 && run + s > target) { owner = r; ahead = run; }
      run += s;
    }
    bool beyond = owner < 0;                                // u outside [0, 1): the last token that has any weight
    if (beyond) owner = last;
    if (rank == owner && warp == 0) {
      int mine = -1;
      run = ahead;
      last = 0;
      for (int i = 0; i < DV_WARPS; ++i) {
        const double s = warp_sum[i];
        if (s > 0.0) last = i;
        if (!beyond && mine < 0 && run + s > target) { mine = i; ahead = run; }
        run += s;
      }
      if (mine < 0) { mine = last; beyond = true; }
      const T* p = p_rows + (size_t)c * V;
      const T* q = q_rows + (size_t)c * V;
      const int x0 = min(cta0 + mine * per_warp, cta1), x1 = min(x0 + per_warp, cta1);
      int found = -1, last_x = -1;
      run = ahead;
      for (int base = x0; base < x1 && found < 0; base += 32) {
        const int x = base + lane;
        double r = 0.0;
        if (x < x1) r = left_of<T, DRAFT>((double)prob(p[x]), DRAFT ? (double)prob(q[x]) : 0.0, x, left);
        double s = r;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double t = __shfl_up_sync(0xffffffffu, s, o);
          if (lane >= o) s += t;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, r > 0.0);
        const uint32_t hit = __ballot_sync(0xffffffffu, r > 0.0 && run + s > target);
        if (some) last_x = base + 31 - __clz(some);
        if (!beyond && hit) found = base + __ffs(hit) - 1;
        run += __shfl_sync(0xffffffffu, s, 31);
      }
      if (lane == 0) a.token[b] = found >= 0 ? found : last_x;
    }
  }
  if (rank == 0) {
    if (tid < N) a.path[(size_t)b * N + tid] = tid < n ? path[tid] : -1;
    if (tid == 0) a.n_accepted[b] = n;
  }
  cluster_sync();                                           // nobody leaves while its sums are being read
}

template <typename T, bool DRAFT>
cudaError_t launch_verify(const VerifyArgs& a, cudaStream_t s) {
  KernelTimer kt("draft_verify", s);
  const cudaError_t e = launch_pdl_cluster(draft_verify_kernel<T, DRAFT>, dim3((unsigned)(a.B * DV_CLUSTER)), dim3(DV_THREADS), 0, s,
                                           true, DV_CLUSTER, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return cudaGetLastError();
}

template <typename T>
cudaError_t launch_verify_as(const VerifyArgs& a, cudaStream_t s) {
  return a.q ? launch_verify<T, true>(a, s) : launch_verify<T, false>(a, s);
}

bool misaligned(const void* p, unsigned by) { return ((uintptr_t)p & (by - 1)) != 0; }

}  // namespace
}  // namespace draft
}  // namespace rattn

using namespace rattn;

extern "C" int rattn_draft_verify(const rattn_verify_params* p, void* stream) {
  using namespace draft;
  if (!p) return RATTN_ERR_NULL_PTR;
  if (p->B < 1 || p->B > (1 << 24) || p->N < 1 || p->N > kMaxNodes || p->V < 1 || p->V > (1 << 30)) return RATTN_ERR_BAD_ARG;
  if (p->dtype != RATTN_BF16 && p->dtype != RATTN_F32) return RATTN_ERR_UNSUPPORTED;
  if (!p->tokens || !p->parents || !p->target_probs || !p->u || !p->path || !p->n_accepted || !p->token) return RATTN_ERR_NULL_PTR;
  if (misaligned(p->tokens, 4) || misaligned(p->parents, 4) || misaligned(p->u, 4) || misaligned(p->path, 4) ||
      misaligned(p->n_accepted, 4) || misaligned(p->token, 4) || misaligned(p->target_probs, 16) || misaligned(p->draft_probs, 16))
    return RATTN_ERR_MISALIGNED;
  VerifyArgs a;
  a.tokens = p->tokens; a.parents = p->parents;
  a.p = p->target_probs; a.q = p->draft_probs;
  a.u = p->u;
  a.path = p->path; a.n_accepted = p->n_accepted; a.token = p->token;
  a.B = p->B; a.N = p->N; a.V = p->V;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = p->dtype == RATTN_BF16 ? launch_verify_as<__nv_bfloat16>(a, s) : launch_verify_as<float>(a, s);
  if (e == cudaSuccess) return RATTN_OK;
  set_last_cuda_error((int)e);
  return RATTN_ERR_CUDA;
}
