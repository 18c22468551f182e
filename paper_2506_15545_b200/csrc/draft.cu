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
// The portable kernel: four warps walk tiles of 32 keys, which they load together into shared memory, a warp for one or four rows.
// A lane forms the scores of its key for the warp's rows, then the lanes hold the features and add the values of those keys that a row
// sees, one by one -- what it does not see is not multiplied, so NaN or infinity there stays there.  It is bound by its
// shared-memory loads and the latency of a tile (16 heads x 64 rows, d = 64, w = 512, fp32: 61 us, 54 with everything
// in L2; there with every lane reading its key's row from global memory 168).
#include <cmath>

#include "draft_internal.h"

namespace rattn {
namespace draft {
namespace {

constexpr int DG_WARPS = 4;

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

// phi(q) . phi(k), fq = phi(q)
template <int D>
__device__ __forceinline__ float phi_dot(const float* fq, const float* k, int phi) {
  float m = -INFINITY, s = 0.f, n = 0.f;
  if (phi == RATTN_PHI_SOFTMAX)
#pragma unroll 8
    for (int i = 0; i < D; ++i) m = fmaxf(m, k[i]);
#pragma unroll 8
  for (int i = 0; i < D; ++i) {
    const float e = phi == RATTN_PHI_SOFTMAX ? expf(k[i] - m) : phi == RATTN_PHI_RELU ? fmaxf(k[i], 0.f) : k[i];
    s += fq[i] * e;
    n += e;
  }
  return phi == RATTN_PHI_SOFTMAX ? s / n : s;
}

template <int D, int RW> struct GenericPlan {             // floats of shared memory
  static constexpr int KS = D + 4;                          // a key's row: lanes 16 bytes apart modulo 128
  static constexpr int K = 0, V = K + 32 * KS, Q = V + 32 * D, F = Q + DG_WARPS * RW * D, END = F + DG_WARPS * RW * D;
};

// RW: rows per warp
template <typename T, int D, int RW>
__global__ void __launch_bounds__(DG_WARPS * 32) draft_generic_kernel(const __grid_constant__ DraftArgs a) {
  using P = GenericPlan<D, RW>;
  constexpr int C = D / 32, ROWS = DG_WARPS * RW;
  extern __shared__ __align__(16) float sm[];
  __shared__ int par[kMaxNodes], depth[kMaxNodes];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int R = a.group * a.N, blocks = (R + ROWS - 1) / ROWS;
  const int z = blockIdx.x / blocks, b = z / a.H_kv, hk = z % a.H_kv, row0 = (blockIdx.x % blocks) * ROWS + warp * RW;
  float* k_s = sm + P::K;
  float* v_s = sm + P::V;
  float* q_s = sm + P::Q + warp * RW * D;
  float* f_s = sm + P::F + warp * RW * D;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");        // the inputs may come from the kernel before
  for (int i = threadIdx.x; i < a.N; i += DG_WARPS * 32) par[i] = a.parents[(size_t)b * a.N + i];
  __syncthreads();
  for (int i = threadIdx.x; i < a.N; i += DG_WARPS * 32) depth[i] = node_depth(par, i);
  __syncthreads();
  const int pos = entry_pos(a, b), w = a.w;
  const RingAge age(pos, w);

  int e[RW];                                                // depth of the row's node; -1: no node
  NodeSet path[RW];
  float m[RW], l[RW], o[RW][C], r[RW][C];
#pragma unroll
  for (int k = 0; k < RW; ++k) {
    const int row = row0 + k, n = min(row, R - 1) / a.group, h = hk * a.group + min(row, R - 1) % a.group;
    e[k] = row < R ? depth[n] : -1;
#pragma unroll
    for (int i = 0; i < kMaxNodes / 32; ++i) path[k].w[i] = 0u;
    if (e[k] >= 0) node_path(par, n, &path[k]);
    const T* qr = static_cast<const T*>(a.q) + node_at(a, b, h, a.H_q, n);
    float x[C], fx[C];
#pragma unroll
    for (int i = 0; i < C; ++i) q_s[k * D + lane + 32 * i] = x[i] = (float)qr[lane + 32 * i];
    if (a.phi == RATTN_PHI_SOFTMAX) {
      float mx = x[0], s = 0.f;
#pragma unroll
      for (int i = 1; i < C; ++i) mx = fmaxf(mx, x[i]);
      mx = wmax(mx);
#pragma unroll
      for (int i = 0; i < C; ++i) s += fx[i] = expf(x[i] - mx);
      s = wsum(s);
#pragma unroll
      for (int i = 0; i < C; ++i) fx[i] /= s;
    } else {
#pragma unroll
      for (int i = 0; i < C; ++i) fx[i] = a.phi == RATTN_PHI_RELU ? fmaxf(x[i], 0.f) : x[i];
    }
    m[k] = -INFINITY;
    l[k] = 0.f;
#pragma unroll
    for (int i = 0; i < C; ++i) {
      f_s[k * D + lane + 32 * i] = fx[i];
      o[k][i] = r[k][i] = 0.f;
    }
  }

  // the keys base .. base + n - 1 (rows `stride` apart) to shared memory; then near / far say how the warp's rows see them
  auto load = [&](const T* kb, const T* vb, size_t stride, int n) {
    __syncthreads();                                        // everybody has read the tile before
    constexpr int PER = D / Vec<T>::N;
#pragma unroll 4
    for (int c = threadIdx.x; c < 32 * PER; c += DG_WARPS * 32) {
      const int j = c / PER, at = (c % PER) * Vec<T>::N;
      if (j >= n) break;
      float x[Vec<T>::N], y[Vec<T>::N];
      Vec<T>::load(kb + j * stride + at, x);
      Vec<T>::load(vb + j * stride + at, y);
#pragma unroll
      for (int i = 0; i < Vec<T>::N; i += 4) {
        *reinterpret_cast<float4*>(k_s + j * P::KS + at + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
        *reinterpret_cast<float4*>(v_s + j * D + at + i) = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
      }
    }
    __syncthreads();
  };
  auto tile = [&](const bool (&near)[RW], const bool (&far)[RW]) {
    float p[RW];
    uint32_t nears[RW], fars[RW], all = 0xffffffffu, any = 0u;
#pragma unroll
    for (int k = 0; k < RW; ++k) {
      nears[k] = __ballot_sync(0xffffffffu, near[k]);
      fars[k] = __ballot_sync(0xffffffffu, far[k]);
      all &= nears[k];
      any |= nears[k] | fars[k];
      p[k] = 0.f;
    }
    if (any == 0u) return;
    if (any >> lane & 1u) {                                  // (rows of the tile behind its last key hold another tile's)
#pragma unroll 4
      for (int i = 0; i < D; i += 4) {
        const float4 x = *reinterpret_cast<const float4*>(k_s + lane * P::KS + i);
#pragma unroll
        for (int k = 0; k < RW; ++k) {
          const float4 q = *reinterpret_cast<const float4*>(q_s + k * D + i);
          p[k] += (q.x * x.x + q.y * x.y) + (q.z * x.z + q.w * x.w);
        }
      }
    }
#pragma unroll
    for (int k = 0; k < RW; ++k) {
      p[k] = near[k] ? p[k] * a.scale : -INFINITY;
      if (nears[k]) {
        const float m_new = fmaxf(m[k], wmax(p[k])), safe = m_new == -INFINITY ? 0.f : m_new, f = expf(m[k] - safe);
        l[k] *= f;
#pragma unroll
        for (int i = 0; i < C; ++i) o[k][i] *= f;
        m[k] = m_new;
        p[k] = near[k] ? expf(p[k] - safe) : 0.f;
        l[k] += wsum(p[k]);
      }
      if (far[k]) p[k] = phi_dot<D>(f_s + k * D, k_s + lane * P::KS, a.phi);
    }
    if (all == 0xffffffffu) {
#pragma unroll 4
      for (int j = 0; j < 32; ++j) {
        float v[C];
#pragma unroll
        for (int i = 0; i < C; ++i) v[i] = v_s[j * D + lane + 32 * i];
#pragma unroll
        for (int k = 0; k < RW; ++k) {
          const float pj = __shfl_sync(0xffffffffu, p[k], j);
#pragma unroll
          for (int i = 0; i < C; ++i) o[k][i] += pj * v[i];
        }
      }
      return;
    }
    for (uint32_t todo = any; todo; todo &= todo - 1) {
      const int j = __ffs(todo) - 1;
      float v[C];
#pragma unroll
      for (int i = 0; i < C; ++i) v[i] = v_s[j * D + lane + 32 * i];
#pragma unroll
      for (int k = 0; k < RW; ++k) {
        const float pj = __shfl_sync(0xffffffffu, p[k], j);
        if (nears[k] >> j & 1u)
#pragma unroll
          for (int i = 0; i < C; ++i) o[k][i] += pj * v[i];
        else if (fars[k] >> j & 1u)
#pragma unroll
          for (int i = 0; i < C; ++i) r[k][i] += pj * v[i];
      }
    }
  };
  const T* kr = static_cast<const T*>(a.k_ring) + (size_t)z * w * D;
  const T* vr = static_cast<const T*>(a.v_ring) + (size_t)z * w * D;
  const int held = min(pos, w);                             // slots 0 .. held-1 hold tokens
  bool near[RW], far[RW];
  for (int s0 = 0; s0 < held; s0 += 32) {
    load(kr + (size_t)s0 * D, vr + (size_t)s0 * D, D, min(32, held - s0));
    const int rank = s0 + lane < held ? age.rank(s0 + lane) : -1;
#pragma unroll
    for (int k = 0; k < RW; ++k) {
      near[k] = e[k] >= 0 && rank >= age.first && rank >= e[k];
      far[k] = rank >= age.first && rank < e[k];
    }
    tile(near, far);
  }
  const size_t step = a.layout == RATTN_LAYOUT_BHTD ? (size_t)D : (size_t)a.H_kv * D;
  for (int j0 = 0; j0 < a.N; j0 += 32) {
    const size_t at = node_at(a, b, hk, a.H_kv, j0);
    load(static_cast<const T*>(a.k) + at, static_cast<const T*>(a.v) + at, step, min(32, a.N - j0));
#pragma unroll
    for (int k = 0; k < RW; ++k) {
      const bool mine = (path[k].w[j0 >> 5] >> lane) & 1u;
      near[k] = mine && e[k] - depth[j0 + lane] <= w;
      far[k] = mine && !near[k];
    }
    tile(near, far);
  }
  const float* S = a.state + (size_t)z * D * D;
#pragma unroll 8
  for (int f = 0; f < D; ++f) {
    float x[C];
#pragma unroll
    for (int i = 0; i < C; ++i) x[i] = S[f * D + lane + 32 * i];
#pragma unroll
    for (int k = 0; k < RW; ++k) {
      const float fq = f_s[k * D + f];
#pragma unroll
      for (int i = 0; i < C; ++i) r[k][i] += fq * x[i];
    }
  }
#pragma unroll
  for (int k = 0; k < RW; ++k) {
    if (e[k] < 0) continue;                                  // (the same for the warp)
    const int n = (row0 + k) / a.group, h = hk * a.group + (row0 + k) % a.group;
#pragma unroll
    for (int i = 0; i < C; ++i) o[k][i] /= l[k];
    const float is = row_inv_rms(o[k], a.eps), ir = row_inv_rms(r[k], a.eps);
    T* out = static_cast<T*>(a.out) + node_at(a, b, h, a.H_q, n);
#pragma unroll
    for (int i = 0; i < C; ++i) {
      const int c = lane + 32 * i;
      const float gs = a.gamma_swa ? a.gamma_swa[(size_t)h * D + c] : 1.f, gr = a.gamma_rla ? a.gamma_rla[(size_t)h * D + c] : 1.f;
      out[c] = (T)(gs * o[k][i] * is + gr * r[k][i] * ir);
    }
  }
}

template <typename T, int D, int RW>
cudaError_t launch_generic_rows(const DraftArgs& a, cudaStream_t s) {
  constexpr int smem = GenericPlan<D, RW>::END * (int)sizeof(float), rows = DG_WARPS * RW;
  cudaError_t e = allow_smem<draft_generic_kernel<T, D, RW>>(smem);
  if (e != cudaSuccess) return e;
  const int blocks = (a.group * a.N + rows - 1) / rows;
  KernelTimer kt("draft_attention", s);
  e = launch_pdl(draft_generic_kernel<T, D, RW>, dim3((unsigned)((long long)a.B * a.H_kv * blocks)), dim3(DG_WARPS * 32), smem, s, true, a);
  if (e != cudaSuccess) return e;
  count_launches(1);
  return cudaGetLastError();
}

// How many CTAs of one row to a warp run at once on the current device, asked of the driver once per device.
template <typename T, int D>
cudaError_t one_row_ctas_at_once(int* n) {
  static std::atomic<int> known[kMaxDevices];
  constexpr int smem = GenericPlan<D, 1>::END * (int)sizeof(float);
  int dev = 0, n_sm = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  if ((*n = known[dev].load(std::memory_order_relaxed)) != 0) return cudaSuccess;
  e = allow_smem<draft_generic_kernel<T, D, 1>>(smem);
  if (e == cudaSuccess) e = sm_count(&n_sm);
  if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(n, draft_generic_kernel<T, D, 1>, DG_WARPS * 32, (size_t)smem);
  *n *= n_sm;
  if (e == cudaSuccess) known[dev].store(*n, std::memory_order_relaxed);
  return e;
}

// A row to a warp while all CTAs of that run at once: a wave takes half of the time of one of four rows to a warp, which share
// the warp's reads of keys and values and win from the second wave on.  One / four, w = 512, fp32: d = 128 (740 CTAs at
// once), 560 CTAs 137 / 201 us, 888 259 / 196, 7680 1373 / 804; d = 64 (1184), 1120 95 / 137, 1536 148 / 116, 7680 591 / 402.
// (w = 100: 1776 CTAs of a head's 192 rows 69 / 85, 7680 231 / 201.)
template <typename T, int D>
cudaError_t launch_generic_as(const DraftArgs& a, cudaStream_t s) {
  int n = 0;
  const cudaError_t e = one_row_ctas_at_once<T, D>(&n);
  if (e != cudaSuccess) return e;
  const long long ctas = (long long)a.B * a.H_kv * ((a.group * a.N + DG_WARPS - 1) / DG_WARPS);
  return ctas <= n ? launch_generic_rows<T, D, 1>(a, s) : launch_generic_rows<T, D, 4>(a, s);
}

bool misaligned(const void* p) { return ((uintptr_t)p & 15u) != 0; }
bool misaligned4(const void* p) { return ((uintptr_t)p & 3u) != 0; }

// Checks what both entry points use and fills the arguments.
int resolve(const rattn_draft_params* p, DraftArgs* a) {
  if (!p) return RATTN_ERR_NULL_PTR;
  if (p->B < 1 || p->H_q < 1 || p->H_kv < 1 || p->N < 1 || p->N > kMaxNodes || p->w < 1) return RATTN_ERR_BAD_ARG;
  if (p->H_q % p->H_kv != 0) return RATTN_ERR_BAD_ARG;
  if (!p->pos_dev && (p->pos < 0 || (long long)p->pos + p->w > 0x7fffffffll)) return RATTN_ERR_BAD_ARG;
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
