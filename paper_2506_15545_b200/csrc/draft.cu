// Speculative decoding: entry points of rattn_draft_attention and rattn_draft_commit, and the portable kernel of the
// attention (any dtype, head size, window and tree; fp32 arithmetic on the CUDA cores).
//
// A node at depth e stands at position pos + e.  With the window's w + 1 tokens and the linear branch behind them, its row is
//
//   o_swa = sum_{j near} softmax(scale q.k_j) v_j,     o_rla = phi(q) S + sum_{j far} (phi(q).phi(k_j)) v_j,
//   y = rmsnorm(o_swa) + rmsnorm(o_rla)
//
// over the ring's tokens and the nodes of its own path: ring tokens of rank >= e and path nodes at most w levels up are
// near, the others far.  S holds everything older and is shared by all nodes: what a sequential decode would have folded
// into it along the path is added in quadratic form (at most as many tokens as the tree is deep).
//
// The portable kernel gives a warp one row.  Blocks of 32 keys: a lane forms the score of its key, then the lanes hold the
// features and add the values of those keys that the row sees, one by one -- what it does not see is not read into a product,
// so NaN or infinity there stays there.
#include <cmath>

#include "draft_internal.h"

namespace rattn {
namespace draft {
namespace {

constexpr int DG_WARPS = 4;

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

template <typename T> struct Vec;              // 16 bytes of a row as fp32
template <> struct Vec<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void load(const float* p, float (&x)[4]) {
    const float4 u = *reinterpret_cast<const float4*>(p);
    x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w;
  }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void load(const __nv_bfloat16* p, float (&x)[8]) {
    const uint4 u = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
};

template <typename T, int D>
__device__ __forceinline__ float dot(const float* q, const T* k) {
  float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 16
  for (int i = 0; i < D; i += Vec<T>::N) {
    float x[Vec<T>::N];
    Vec<T>::load(k + i, x);
#pragma unroll
    for (int j = 0; j < Vec<T>::N; ++j) s[j & 3] += q[i + j] * x[j];
  }
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// phi(q) . phi(k), fq = phi(q)
template <typename T, int D>
__device__ __forceinline__ float phi_dot(const float* fq, const T* k, int phi) {
  if (phi == RATTN_PHI_IDENTITY) return dot<T, D>(fq, k);
  float m = -INFINITY, s = 0.f, n = 0.f;
  if (phi == RATTN_PHI_SOFTMAX)
#pragma unroll 4
    for (int i = 0; i < D; i += Vec<T>::N) {
      float x[Vec<T>::N];
      Vec<T>::load(k + i, x);
#pragma unroll
      for (int j = 0; j < Vec<T>::N; ++j) m = fmaxf(m, x[j]);
    }
#pragma unroll 4
  for (int i = 0; i < D; i += Vec<T>::N) {
    float x[Vec<T>::N];
    Vec<T>::load(k + i, x);
#pragma unroll
    for (int j = 0; j < Vec<T>::N; ++j) {
      const float e = phi == RATTN_PHI_SOFTMAX ? expf(x[j] - m) : fmaxf(x[j], 0.f);
      s += fq[i + j] * e;
      n += e;
    }
  }
  return phi == RATTN_PHI_SOFTMAX ? s / n : s;
}

template <typename T, int D>
__global__ void __launch_bounds__(DG_WARPS * 32) draft_generic_kernel(const __grid_constant__ DraftArgs a) {
  constexpr int C = D / 32;
  __shared__ __align__(16) float q_s[DG_WARPS][D];
  __shared__ __align__(16) float f_s[DG_WARPS][D];
  __shared__ int par[kMaxNodes], depth[kMaxNodes];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = a.group * a.N, blocks = (R + DG_WARPS - 1) / DG_WARPS;
  const int z = blockIdx.x / blocks, b = z / a.H_kv, hk = z % a.H_kv;
  const int row = (blockIdx.x % blocks) * DG_WARPS + warp, n = row / a.group, h = hk * a.group + row % a.group;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");        // the inputs may come from the kernel before
  for (int i = threadIdx.x; i < a.N; i += DG_WARPS * 32) par[i] = a.parents[(size_t)b * a.N + i];
  __syncthreads();
  for (int i = threadIdx.x; i < a.N; i += DG_WARPS * 32) depth[i] = node_depth(par, i);
  __syncthreads();
  const int e = row < R ? depth[n] : -1;
  if (e < 0) return;
  NodeSet path;
  node_path(par, n, &path);
  const int pos = entry_pos(a, b), w = a.w;
  const RingAge age(pos, w);

  const T* qr = static_cast<const T*>(a.q) + node_at(a, b, h, a.H_q, n);
  float x[C], fx[C];
#pragma unroll
  for (int i = 0; i < C; ++i) q_s[warp][lane + 32 * i] = x[i] = (float)qr[lane + 32 * i];
  if (a.phi == RATTN_PHI_SOFTMAX) {
    float m = x[0], s = 0.f;
#pragma unroll
    for (int i = 1; i < C; ++i) m = fmaxf(m, x[i]);
    m = wmax(m);
#pragma unroll
    for (int i = 0; i < C; ++i) s += fx[i] = expf(x[i] - m);
    s = wsum(s);
#pragma unroll
    for (int i = 0; i < C; ++i) fx[i] /= s;
  } else {
#pragma unroll
    for (int i = 0; i < C; ++i) fx[i] = a.phi == RATTN_PHI_RELU ? fmaxf(x[i], 0.f) : x[i];
  }
#pragma unroll
  for (int i = 0; i < C; ++i) f_s[warp][lane + 32 * i] = fx[i];
  __syncwarp();

  float m = -INFINITY, l = 0.f, o[C], r[C];
#pragma unroll
  for (int i = 0; i < C; ++i) o[i] = r[i] = 0.f;
  // keys base + lane * stride of up to 32: near / far say which of them the row sees how
  auto block = [&](const T* kb, const T* vb, size_t stride, bool near, bool far) {
    const uint32_t nears = __ballot_sync(0xffffffffu, near), fars = __ballot_sync(0xffffffffu, far);
    if ((nears | fars) == 0u) return;
    float p = near ? dot<T, D>(q_s[warp], kb + lane * stride) * a.scale : -INFINITY;
    if (nears) {
      const float m_new = fmaxf(m, wmax(p)), safe = m_new == -INFINITY ? 0.f : m_new, f = expf(m - safe);
      l *= f;
#pragma unroll
      for (int i = 0; i < C; ++i) o[i] *= f;
      m = m_new;
      p = near ? expf(p - safe) : 0.f;
      l += wsum(p);
    }
    if (far) p = phi_dot<T, D>(f_s[warp], kb + lane * stride, a.phi);
    if (nears == 0xffffffffu) {                              // all of them near: eight values on their way at a time
      for (int j0 = 0; j0 < 32; j0 += 8) {
        T vv[8][C];
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int i = 0; i < C; ++i) vv[j][i] = vb[(j0 + j) * stride + lane + 32 * i];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float pj = __shfl_sync(0xffffffffu, p, j0 + j);
#pragma unroll
          for (int i = 0; i < C; ++i) o[i] += pj * (float)vv[j][i];
        }
      }
      return;
    }
    for (uint32_t todo = nears | fars; todo; todo &= todo - 1) {
      const int j = __ffs(todo) - 1;
      const float pj = __shfl_sync(0xffffffffu, p, j);
      const T* vr = vb + j * stride;
      const bool is_near = (nears >> j) & 1u;
#pragma unroll
      for (int i = 0; i < C; ++i) {
        const float vv = (float)vr[lane + 32 * i];
        if (is_near) o[i] += pj * vv;
        else r[i] += pj * vv;
      }
    }
  };
  const T* kr = static_cast<const T*>(a.k_ring) + (size_t)z * w * D;
  const T* vr = static_cast<const T*>(a.v_ring) + (size_t)z * w * D;
  const int held = min(pos, w);                             // slots 0 .. held-1 hold tokens
  for (int s0 = 0; s0 < held; s0 += 32) {
    const int rank = s0 + lane < held ? age.rank(s0 + lane) : -1;
    block(kr + (size_t)s0 * D, vr + (size_t)s0 * D, D, rank >= age.first && rank >= e, rank >= age.first && rank < e);
  }
  const size_t step = a.layout == RATTN_LAYOUT_BHTD ? (size_t)D : (size_t)a.H_kv * D;
  for (int j0 = 0; j0 < a.N; j0 += 32) {
    const size_t at = node_at(a, b, hk, a.H_kv, j0);
    const bool mine = (path.w[j0 >> 5] >> lane) & 1u, near = mine && e - depth[j0 + lane] <= w;
    block(static_cast<const T*>(a.k) + at, static_cast<const T*>(a.v) + at, step, near, mine && !near);
  }
  const float* S = a.state + (size_t)z * D * D;
#pragma unroll 16
  for (int f = 0; f < D; ++f) {
    const float fq = f_s[warp][f];
#pragma unroll
    for (int i = 0; i < C; ++i) r[i] += fq * S[f * D + lane + 32 * i];
  }
  float so = 0.f, sr = 0.f;
#pragma unroll
  for (int i = 0; i < C; ++i) {
    o[i] /= l;
    so += o[i] * o[i];
    sr += r[i] * r[i];
  }
  const float is = rsqrtf(wsum(so) / D + a.eps), ir = rsqrtf(wsum(sr) / D + a.eps);
  T* out = static_cast<T*>(a.out) + node_at(a, b, h, a.H_q, n);
#pragma unroll
  for (int i = 0; i < C; ++i) {
    const int c = lane + 32 * i;
    const float gs = a.gamma_swa ? a.gamma_swa[(size_t)h * D + c] : 1.f, gr = a.gamma_rla ? a.gamma_rla[(size_t)h * D + c] : 1.f;
    out[c] = (T)(gs * o[i] * is + gr * r[i] * ir);
  }
}

template <typename T, int D>
cudaError_t launch_generic_as(const DraftArgs& a, cudaStream_t s) {
  const int blocks = (a.group * a.N + DG_WARPS - 1) / DG_WARPS;
  KernelTimer kt("draft_attention", s);
  const cudaError_t e = launch_pdl(draft_generic_kernel<T, D>, dim3((unsigned)((long long)a.B * a.H_kv * blocks)),
                                   dim3(DG_WARPS * 32), 0, s, true, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return cudaGetLastError();
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
bool misaligned4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

// Checks what both entry points use and fills the arguments.
int resolve(const rattn_draft_params* p, DraftArgs* a) {
  if (!p) return RATTN_ERR_NULL_PTR;
  if (p->B < 1 || p->H_q < 1 || p->H_kv < 1 || p->N < 1 || p->N > kMaxNodes || p->w < 1) return RATTN_ERR_BAD_ARG;
  if (p->H_q % p->H_kv != 0) return RATTN_ERR_BAD_ARG;
  if (!p->pos_dev && (p->pos < 0 || (long long)p->pos + kMaxNodes + p->w > 0x7fffffffll)) return RATTN_ERR_BAD_ARG;
  // row and slot counts stay below 2^31
  if ((long long)p->B * p->H_q * p->N >= (1ll << 31) || (long long)p->B * p->H_kv * p->w >= (1ll << 31) ||
      (long long)p->B * p->H_kv >= (1ll << 28))
    return RATTN_ERR_BAD_ARG;
  if (p->d != 64 && p->d != 128) return RATTN_ERR_UNSUPPORTED;
  if (p->dtype != RATTN_BF16 && p->dtype != RATTN_F32) return RATTN_ERR_UNSUPPORTED;
  if (p->feature_map < RATTN_PHI_SOFTMAX || p->feature_map > RATTN_PHI_IDENTITY) return RATTN_ERR_UNSUPPORTED;
  if (p->layout != RATTN_LAYOUT_BHTD && p->layout != RATTN_LAYOUT_BTHD) return RATTN_ERR_UNSUPPORTED;
  if (!p->k || !p->v || !p->k_ring || !p->v_ring || !p->state) return RATTN_ERR_NULL_PTR;
  if (misaligned(p->k) || misaligned(p->v) || misaligned(p->k_ring) || misaligned(p->v_ring) || misaligned(p->state) ||
      misaligned4(p->pos_dev))
    return RATTN_ERR_MISALIGNED;
  a->q = p->q; a->k = p->k; a->v = p->v; a->out = p->out;
  a->parents = p->parents;
  a->k_ring = p->k_ring; a->v_ring = p->v_ring; a->state = p->state;
  a->gamma_swa = p->gamma_swa; a->gamma_rla = p->gamma_rla;
  a->pos_dev = p->pos_dev; a->path = p->path; a->n_accepted = p->n_accepted;
  a->B = p->B; a->H_q = p->H_q; a->H_kv = p->H_kv; a->N = p->N; a->d = p->d; a->w = p->w;
  a->group = p->H_q / p->H_kv;
  a->dtype = p->dtype; a->phi = p->feature_map; a->layout = p->layout; a->pos = p->pos; a->flags = p->flags;
  a->scale = p->scale; a->eps = p->eps;
  return RATTN_OK;
}

int result(cudaError_t e) {
  if (e == cudaSuccess) return RATTN_OK;
  set_last_cuda_error((int)e);
  return RATTN_ERR_CUDA;
}

}  // namespace

cudaError_t launch_generic(const DraftArgs& a, cudaStream_t s) {
  if (a.dtype == RATTN_BF16)
    return a.d == 128 ? launch_generic_as<__nv_bfloat16, 128>(a, s) : launch_generic_as<__nv_bfloat16, 64>(a, s);
  return a.d == 128 ? launch_generic_as<float, 128>(a, s) : launch_generic_as<float, 64>(a, s);
}

}  // namespace draft
}  // namespace rattn

using namespace rattn;

extern "C" {

int rattn_draft_attention(const rattn_draft_params* p, void* stream) {
  draft::DraftArgs a;
  const int rc = draft::resolve(p, &a);
  if (rc != RATTN_OK) return rc;
  if (!(p->eps > 0.f) || std::isinf(p->eps) || !std::isfinite(p->scale)) return RATTN_ERR_BAD_ARG;
  if (!p->q || !p->out || !p->parents) return RATTN_ERR_NULL_PTR;
  if (draft::misaligned(p->q) || draft::misaligned(p->out) || draft::misaligned(p->gamma_swa) ||
      draft::misaligned(p->gamma_rla) || draft::misaligned4(p->parents))
    return RATTN_ERR_MISALIGNED;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  return draft::result(draft::tc_applies(a) ? draft::launch_tc(a, s) : draft::launch_generic(a, s));
}

int rattn_draft_commit(const rattn_draft_params* p, void* stream) {
  if (!p) return RATTN_ERR_NULL_PTR;
  rattn_draft_params heads = *p;                            // the query heads play no part
  heads.H_q = p->H_kv;
  draft::DraftArgs a;
  const int rc = draft::resolve(&heads, &a);
  if (rc != RATTN_OK) return rc;
  if (!p->path || !p->n_accepted) return RATTN_ERR_NULL_PTR;
  if (draft::misaligned4(p->path) || draft::misaligned4(p->n_accepted)) return RATTN_ERR_MISALIGNED;
  return draft::result(draft::launch_commit(a, reinterpret_cast<cudaStream_t>(stream)));
}

int rattn_draft_status(void* stream) {
  cudaError_t e = cudaSuccess;
  const int word = draft::tc_status(reinterpret_cast<cudaStream_t>(stream), &e);
  if (e != cudaSuccess) return draft::result(e);
  return word == 0 ? RATTN_OK : RATTN_ERR_TIMEOUT;
}

}  // extern "C"
