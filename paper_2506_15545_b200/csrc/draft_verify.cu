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
// nothing but the partial sums passes between them, through distributed shared memory.  r is never stored: q being at least 0,
// max(max(p - a q, 0) - b q, 0) = max(p - (a + b) q, 0), so r after any number of rejections is formed from p, q and the sum
// of their Z.  A thread asks for 64 bytes or more of either row before it uses the first of them.  Sums, r and comparisons are
// fp64: the drawn token is an index, and in fp32 the running sum over 10^5 tokens of 10^-5 would be off by as much as
// their probabilities.


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

__device__ __forceinline__ float prob(float f) { return f > 0.f ? f : 0.f; }      // negative and NaN count as 0

// 16 bytes of a row.  A row of a vocabulary of any size may start anywhere, so a row is walked from the 16-byte boundary at or
// before its start (what lies there is the row ahead of it) and its last few probabilities are read one by one.
template <typename T> struct Probs;
template <> struct Probs<float> {
  static constexpr int N = 4;
  float4 raw;
  __device__ __forceinline__ void load(const float* p) { raw = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void load_some(const float* p, int n) {
    raw = make_float4(n > 0 ? p[0] : 0.f, n > 1 ? p[1] : 0.f, n > 2 ? p[2] : 0.f, 0.f);
  }
  __device__ __forceinline__ float at(int i) const { return prob(i == 0 ? raw.x : i == 1 ? raw.y : i == 2 ? raw.z : raw.w); }
};
template <> struct Probs<__nv_bfloat16> {
  static constexpr int N = 8;
  uint4 raw;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { raw = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load_some(const __nv_bfloat16* p, int n) {
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < 7; ++i)
      if (i < n) w[i >> 1] |= (uint32_t)__bfloat16_as_ushort(p[i]) << (16 * (i & 1));
    raw = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ float at(int i) const {
    const uint32_t w = i < 2 ? raw.x : i < 4 ? raw.y : i < 6 ? raw.z : raw.w;
    return prob(__uint_as_float((i & 1) ? w & 0xffff0000u : w << 16));
  }
};

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
  int n;                         // without a drafter's row: tokens taken out
  int x[kMaxNodes];
};
__device__ __forceinline__ bool taken_out(const Left& l, int x) {
  for (int i = 0; i < l.n; ++i)
    if (l.x[i] == x) return true;
  return false;
}

template <typename T, bool DRAFT>
__global__ void __launch_bounds__(DV_THREADS, 2) draft_verify_kernel(const __grid_constant__ VerifyArgs a) {
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
    pt[tid] = real ? (double)prob((float)p_rows[(size_t)up * V + x]) : 0.0;
    qt[tid] = DRAFT ? (real ? (double)prob((float)q_rows[(size_t)up * V + x]) : 0.0) : 1.0;
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
  // Runs of the vocabulary: this CTA's, this warp's, in steps of 32 lanes x VEC tokens.
  // (Places in a row: token x of node c's row is at place x + shift, shift = c V modulo VEC.)
  constexpr int VEC = Probs<T>::N, STEP = 32 * VEC, AHEAD = 4;
  const int per_warp = (V + VEC - 1 + DV_CLUSTER * DV_WARPS * STEP - 1) / (DV_CLUSTER * DV_WARPS * STEP) * STEP, per_cta = per_warp * DV_WARPS;
  const int w0 = rank * per_cta + warp * per_warp;
  int turn = 0;
  double gone = 0.0;                                        // the sum of Z over the rejections that count
  auto shift_of = [&](int c) { return (int)(((size_t)b * N + c) * V % VEC); };
  // the VEC probabilities at place k of a row; row: its place 0
  auto fetch = [&](Probs<T>* v, const T* row, int k, int end) {
    if (k + VEC <= end) v->load(row + k);
    else v->load_some(row + k, end - k);
  };
  // r of VEC tokens from x on, after rejections of `taken` in all.  edge: some of them may lie in front of the row or behind it,
  // where there is none.
  auto left_of = [&](const Probs<T>& p, const Probs<T>& q, int x, double taken, bool check, double (&r)[VEC], bool edge) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      r[i] = (double)p.at(i);
      if (DRAFT) {
        r[i] = r[i] - taken * (double)q.at(i);
        const int hi = __double2hiint(r[i]), keep = ~(hi >> 31);       // max(r, 0)
        r[i] = __hiloint2double(hi & keep, __double2loint(r[i]) & keep);
      } else if (check && taken_out(left, x + i)) {
        r[i] = 0.0;
      }
      if (edge && (unsigned)(x + i) >= (unsigned)V) r[i] = 0.0;
    }
  };
  // whether one of the tokens x .. x + n - 1 has been taken out
  auto any_out = [&](int x, int n) {
    bool any = false;
    if (!DRAFT)
      for (int i = 0; i < left.n; ++i) any |= (unsigned)(left.x[i] - x) < (unsigned)n;
    return any;
  };
  // Sum of r over the vocabulary.  Leaves the warps' sums in warp_sum and the CTAs' in cta_sum[turn - 1].
  auto total = [&](int c, double taken) -> double {
    const int shift = shift_of(c), end = V + shift, w1 = min(w0 + per_warp, end);
    const T* p = p_rows + (size_t)c * V - shift;
    const T* q = q_rows + (size_t)c * V - shift;
    double s = 0.0;
    auto add = [&](const Probs<T>& pv, const Probs<T>& qv, int base, bool edge) {
      double r[VEC];
      left_of(pv, qv, base + lane * VEC - shift, taken, any_out(base - shift, STEP), r, edge);
#pragma unroll
      for (int i = 0; i < VEC; i += 4) s += (r[i] + r[i + 1]) + (r[i + 2] + r[i + 3]);
    };
    auto some = [&](int base) {                             // a step at an end of the row
      Probs<T> pv, qv;
      fetch(&pv, p, base + lane * VEC, end);
      if (DRAFT) fetch(&qv, q, base + lane * VEC, end);
      add(pv, qv, base, true);
    };
    int base = w0;
    if (base == 0 && shift > 0 && w1 > 0) {
      some(0);
      base = STEP;
    }
#pragma unroll 1
    for (; base + AHEAD * STEP <= w1; base += AHEAD * STEP) {          // whole vectors
      Probs<T> pv[AHEAD], qv[AHEAD];
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) {
        pv[j].load(p + base + j * STEP + lane * VEC);
        if (DRAFT) qv[j].load(q + base + j * STEP + lane * VEC);
      }
#pragma unroll
      for (int j = 0; j < AHEAD; ++j) add(pv[j], qv[j], base + j * STEP, false);
    }
#pragma unroll 1
    for (; base < w1; base += STEP) some(base);
    s = wsum(s);
    if (lane == 0) warp_sum[warp] = s;
    __syncthreads();
    if (warp == 0) {
      double t = lane < DV_WARPS ? warp_sum[lane] : 0.0;
      t = wsum(t);
      if (lane == 0) cta_sum[turn & 1] = t;
    }
    cluster_sync();
    double part[DV_CLUSTER], t = 0.0;
#pragma unroll
    for (int r = 0; r < DV_CLUSTER; ++r) part[r] = ld_cluster(&cta_sum[turn & 1], r);
#pragma unroll
    for (int r = 0; r < DV_CLUSTER; ++r) t += part[r];
    ++turn;
    return t;
  };

  constexpr double kTiny = 1.0 / (double)(1ull << 40);
  int c = 0, n = 1;
  double Z = 1.0, sum = 0.0;
  bool pending = false, summed = false;                     // summed: the last pass was over r as it is now
  // a rejection whose sum has not been formed
  auto settle = [&]() {
    const double s = total(c, gone + Z);
    const bool counts = s > kTiny * Z;
    if (counts) {
      gone += Z;
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
    const double r = DRAFT ? fmax(pt[i] - gone * qt[i], 0.0) : taken_out(left, x) ? 0.0 : pt[i];
    if ((double)u_s[i] * qt[i] * Z < r) {
      c = i;
      Z = 1.0;
      gone = 0.0;
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
  if (!summed) sum = total(c, gone);
  if (!(sum > 0.0) && (gone > 0.0 || left.n > 0)) {         // nothing left: the row as it is given
    __syncthreads();
    if (tid == 0) left.n = 0;
    __syncthreads();
    gone = 0.0;
    sum = total(c, 0.0);
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
      const int shift = shift_of(c), end = V + shift;
      const T* p = p_rows + (size_t)c * V - shift;
      const T* q = q_rows + (size_t)c * V - shift;
      const int k0 = rank * per_cta + mine * per_warp, k1 = min(k0 + per_warp, end);
      int found = -1, last_x = -1;
      run = ahead;
      for (int base = k0; base < k1 && found < 0; base += STEP) {
        const int k = base + lane * VEC;
        Probs<T> pv, qv;
        fetch(&pv, p, k, end);
        if (DRAFT) fetch(&qv, q, k, end);
        double r[VEC], s = 0.0;
        left_of(pv, qv, k - shift, gone, any_out(base - shift, STEP), r, true);
        bool mine_any = false;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          s += r[i];
          mine_any |= r[i] > 0.0;
        }
        double upto = s;                                     // of the lanes up to this one
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double t = __shfl_up_sync(0xffffffffu, upto, o);
          if (lane >= o) upto += t;
        }
        int last_i = -1, hit_i = -1;
        double t = run + (upto - s);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          t += r[i];
          if (r[i] > 0.0) last_i = i;
          if (hit_i < 0 && r[i] > 0.0 && t > target) hit_i = i;
        }
        const uint32_t some = __ballot_sync(0xffffffffu, mine_any), hit = __ballot_sync(0xffffffffu, hit_i >= 0);
        if (some) {
          const int from = 31 - __clz(some);
          last_x = base - shift + from * VEC + __shfl_sync(0xffffffffu, last_i, from);
        }
        if (!beyond && hit) {
          const int from = __ffs(hit) - 1;
          found = base - shift + from * VEC + __shfl_sync(0xffffffffu, hit_i, from);
        }
        run += __shfl_sync(0xffffffffu, upto, 31);
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
