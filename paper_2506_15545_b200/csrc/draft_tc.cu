// Attention of a tree of drafts for bf16, d = 128 and a positive scale (sm_100a: TMA + tcgen05 + TMEM).
//
// The rows of a K/V head are its group's query heads at all nodes, R = group * N of them (node by node, so that neighbouring
// rows share their keys); a CTA takes up to 128.  It walks the ring's slots and then the tree's nodes in tiles of 64 keys:
//
//   4 row warps   (thread = row = TMEM lane) online softmax straight out of TMEM; the weights go back over their scores as a
//                 bf16 pair, leading part and remainder, and P V runs over both: 16 bits of every weight, no restriction on v
//   score warp    S = Q K^T
//   MMA warp      O += P V (A operand from TMEM), then the linear branch's products
//   loader warp   TMA: K and V tiles through a ring of five 16 KB slots
//   helper warp   clears V rows that belong to no token or node (0 * NaN), and finds nodes whose values are not finite
//
// Masks: a row at depth e does not see the e oldest slots (as intervals of slots, in the tiles that hold some of them) and
// sees the nodes of its own path (128 bits, from a walk up its parents).
//
// Linear branch, O_rla = phi(Q) S + (phi(Q) phi(K_far)^T masked) V_far: phi(Q) replaces Q without its normalisation (which the
// rows apply at the end) as a bf16 pair, S is split likewise, and three products give 16 bits of both; K_far are the at
// most 127 tokens that have left some row's window (slots of rank < depth; nodes more than w levels up), gathered into a tile.
// The window output waits in TMEM meanwhile, where the far keys' scores and weights leave it 96 of its 128 columns: each value is
// rounded to the upper 24 bits of its fp32 form, off by 2^-17 of itself whatever the row's size, eps or gain.  y leaves through
// shared memory, a warp per row, where gains are read once per row and coalesced.
//
// Few heads (B H_kv row tiles that find room as clusters): a cluster of CTAs shares the tiles of keys and the features of S; the partial
// outputs (fp32) meet through distributed shared memory, a warp per row.
//
// A node with a value that is not finite is cleared in the tile (its zero weight would spread it over all rows) and makes the
// rows that see it NaN.
#include "draft_internal.h"
#include "tc_common.cuh"

namespace rattn {
namespace draft {
namespace {

using namespace ptx;
using namespace tc;

constexpr int FAR = 32;                                      // far keys that are taken at a time
constexpr int DA_NS = 5, DA_THREADS = 256, DA_CLUSTER_ROWS = 96;
constexpr int DA_OFF_RING = TILE_BYTES;
constexpr int DA_OFF_BARS = DA_OFF_RING + DA_NS * HT_BYTES;
constexpr int DA_SMEM = DA_OFF_BARS + 1024;                  // 115,712 bytes: two CTAs share the SM's 228 KB
constexpr int DA_OFF_OX = DA_SMEM;                           // cluster: [rows][128] fp32 of the window branch, of the linear one
constexpr int DA_OFF_STAT = DA_OFF_OX + 2 * DA_CLUSTER_ROWS * 512;
constexpr int DA_SMEM_CLUSTER = DA_OFF_STAT + 2 * DA_CLUSTER_ROWS * 4;
constexpr float LOG2E = 1.4426950408889634f;

__device__ int g_draft_status;           // RATTN_ERR_TIMEOUT once a bounded wait has expired

struct Bars {
  uint64_t full[DA_NS], free_[DA_NS], s_full[2], p_ready[2], pv_done[2], q_full, scored, o_full, done, drain;
  // The (at most three) V tiles that are cleaned: landed, cleaned.  Their landing has barriers of its own, because the
  // helpers follow these uses of the slots alone and a wait by parity cannot skip a phase.
  uint64_t landed[3], clean[3];
  uint32_t tmem_base;
  int abort;
  uint32_t bad[kMaxNodes / 32];          // nodes with a value that is not finite
  signed char depth[kMaxNodes];          // -1: no node
  int n_far_node, deepest;
  union {
    struct {
      signed char par[kMaxNodes];        // -2: no node
      short far_node[kMaxNodes];         // nodes that some row has more than w levels up
    };
    float window_scale[TILE];            // the output: what a row of the window branch is to be multiplied by
  };
};
static_assert(sizeof(Bars) <= DA_SMEM - DA_OFF_BARS, "control block");

struct TcArgs {
  DraftArgs d;
  int row_tiles, rows_per_tile, cluster;
  float scale_log2, inv_group;
  int debug_wait;                        // debug build only, 1: an arrival is left out, 2: a wait counts as run out
};
struct alignas(64) TcMaps {
  CUtensorMap k_ring, v_ring;            // [B*H_kv, w, 128], box 64 columns x 64 slots
  UMap k, v;                             // the nodes' tensors, box 64 columns x 64 nodes
};

__device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1; }   // bits < n
__device__ __forceinline__ bool not_finite(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }

// Order of the loads: K_0, K_1, V_0, K_2, V_1, ..., V_{n-1} -- that of their use.
__device__ __forceinline__ int use_k(int t) { return t == 0 ? 0 : 2 * t - 1; }
__device__ __forceinline__ int use_v(int t, int n) { return t < n - 1 ? 2 * t + 2 : 2 * n - 1; }

// barrier among n threads (id)
__device__ __forceinline__ void named_sync(int id, int n) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(n) : "memory"); }
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_addr(const void* p, int rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ float ld_cluster(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

// Four floats in three words, each with the upper 24 of its bits (rounded: off by 2^-17 of the value at most): three in a word's upper
// bytes, and the fourth's bytes in the lower ones.  (A NaN may come back as a number; its row's scale is NaN, too.)
__device__ __forceinline__ void pack24(const float* x, uint32_t* w0, uint32_t* w1, uint32_t* w2) {
  uint32_t u[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __float_as_uint(x[i]) + 0x80u;
  *w0 = __byte_perm(u[0], u[3], 0x3217);
  *w1 = __byte_perm(u[1], u[3], 0x3216);
  *w2 = __byte_perm(u[2], u[3], 0x3215);
}
__device__ __forceinline__ float4 unpack24(uint32_t w0, uint32_t w1, uint32_t w2) {
  const uint32_t last = __byte_perm(__byte_perm(w0, w1, 0x0400), w2, 0x3244);
  return make_float4(__uint_as_float(w0 & 0xffffff00u), __uint_as_float(w1 & 0xffffff00u), __uint_as_float(w2 & 0xffffff00u),
                     __uint_as_float(last & 0xffffff00u));
}
// Two floats as a word of leading parts (the upper halves of their bits, a byte permutation instead of a conversion) and one
// of remainders, which a conversion rounds: off by 2^-16 of the value at most.
__device__ __forceinline__ void split2(float a, float b, uint32_t* hi, uint32_t* lo) {
  const uint32_t x = __float_as_uint(a), y = __float_as_uint(b);
  *hi = __byte_perm(x, y, 0x7632);
  const float2 r = __ffma2_rn(make_float2(__uint_as_float(x & 0xffff0000u), __uint_as_float(y & 0xffff0000u)), make_float2(-1.f, -1.f),
                              make_float2(a, b));
  *lo = pack_bf16(r.x, r.y);
}
// byte offset of 16-byte chunk c (0 .. 15) of row r in a [128 x 128] bf16 tile (two swizzled halves), and in a half tile
__device__ __forceinline__ uint32_t at_tile(int r, int c) { return (uint32_t)((c >> 3) * HALF_BYTES + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }
__device__ __forceinline__ uint32_t at_half(int r, int c) { return (uint32_t)((c >> 3) * HT_HALF + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }
// an fp32 row of the cluster's exchange: 32 chunks of 16 bytes, permuted so that lanes on different rows meet different banks
__device__ __forceinline__ uint32_t at_ox(int r, int c) { return (uint32_t)(r * 512 + ((c ^ (r & 31)) << 4)); }

// x / G for 0 <= x < 2^21 without an integer division ((x + 0.5) / G is at least 0.5 / G away from an integer, and two
// roundings by 2^-24 of it are less)
__device__ __forceinline__ int small_div(int x, float inv) { return __float2int_rd(((float)x + 0.5f) * inv); }
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src, bool live) {   // zero where not live
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(live ? 16 : 0) : "memory");
}

// What a CTA works on.
struct Item {
  int b, hk, z, rank, row0, rows;        // rows row0 .. row0 + rows - 1 of K/V head hk of entry b
  int pos, held, n_ring, t0, nt;         // slots that hold tokens, their tiles; this CTA's tiles: ring tiles, then node tiles
};
__device__ __forceinline__ Item make_item(const TcArgs& a, int rank) {
  const DraftArgs& d = a.d;
  Item i;
  const int item = blockIdx.x / a.cluster, rt = item % a.row_tiles;
  i.z = item / a.row_tiles;
  i.b = i.z / d.H_kv;
  i.hk = i.z - i.b * d.H_kv;
  i.rank = rank;
  i.row0 = rt * a.rows_per_tile;
  i.rows = min(a.rows_per_tile, d.group * d.N - i.row0);
  i.pos = entry_pos(d, i.b);
  i.held = min(i.pos, d.w);
  i.n_ring = (i.held + 63) >> 6;
  const int all = i.n_ring + ((d.N + 63) >> 6);
  i.t0 = (int)((long long)all * rank / a.cluster);
  i.nt = (int)((long long)all * (rank + 1) / a.cluster) - i.t0;
  return i;
}
// V tile T may hold rows that are no tokens, or (nodes) values that are not finite
__device__ __forceinline__ int first_unclean(const Item& it) { return max(it.t0, it.n_ring - ((it.held & 63) ? 1 : 0)); }
__device__ __forceinline__ bool needs_cleaning(const Item& it, int T) { return T >= first_unclean(it); }

// the use i of the ring of slots (whole warp)
__device__ __forceinline__ void load_use(const TcMaps& m, const Item& it, unsigned char* smem, Bars* bars, int i) {
  const bool is_v = i == 2 * it.nt - 1 || (i > 0 && (i & 1) == 0);
  const int t = i == 0 ? 0 : i == 2 * it.nt - 1 ? it.nt - 1 : is_v ? (i - 2) >> 1 : (i + 1) >> 1, T = it.t0 + t;
  const int slot = i % DA_NS;
  unsigned char* dst = smem + DA_OFF_RING + slot * HT_BYTES;
  uint64_t* bar = &bars->full[slot];
  if (is_v && needs_cleaning(it, T)) {
    mbar_arrive_expect_tx(bar, 0);                           // (the phases of the slot's barrier go on)
    bar = &bars->landed[T - first_unclean(it)];
  }
  mbar_arrive_expect_tx(bar, HT_BYTES);
  if (T < it.n_ring) load_half_tile(dst, is_v ? &m.v_ring : &m.k_ring, bar, 64 * T, it.z);
  else load_half_tile(dst, is_v ? &m.v : &m.k, bar, 64 * (T - it.n_ring), it.z);
}

// S = Q K^T of one tile of 64 keys, D[128 x 64]
__device__ __forceinline__ void mma_scores(uint32_t d, uint32_t q, uint32_t k) { mma_k_kh(d, q, k); }
// O += (hi + lo) V: A from TMEM, hi in columns from 0 on, lo from `lo` on
__device__ __forceinline__ void mma_weights(uint32_t o, uint32_t p, int lo, uint32_t v, bool acc, int steps) {
  constexpr uint32_t idesc = instr_desc(128, 128, 0, 1);
  const uint64_t v0 = mnmajor_base_h(v);
#pragma unroll
  for (int part = 0; part < 2; ++part)
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (k < steps) mma_bf16_ts(o, p + lo * part + 8 * k, v0 + kstep_mn(k), idesc, (acc || part > 0 || k > 0) ? 1u : 0u);
}

// ---------------------------------------------------------------------------------------------- window loop, by role

// Scores and products are issued by two warps: with its waits (some 300 cycles each, satisfied or not), its issue slots (65 per
// instruction) and its commits one warp took 2.1 - 2.4k cycles a tile, the row warps take 1.5k.
// A role whose wait has run out issues nothing more: what it would overwrite or read may still be on its way.
__device__ void window_scores(const Item& it, unsigned char* smem, Bars* bars, uint32_t tS) {
  const uint32_t sQ = smem_u32(smem), sR = sQ + DA_OFF_RING;
  bool ok = mbar_wait_warp(&bars->q_full, 0u, &bars->abort);
  for (int t = 0; t < it.nt && ok; ++t) {
    const int i = use_k(t), slot = i % DA_NS;
    ok = mbar_wait_warp(&bars->full[slot], (uint32_t)(i / DA_NS) & 1u, &bars->abort);
    if (ok && t >= 2) ok = mbar_wait_warp(&bars->pv_done[t & 1], (uint32_t)((t - 2) >> 1) & 1u, &bars->abort);     // its weights lay there
    if (!ok) break;
    tc_fence_after();
    mma_scores(tS + 64 * (t & 1), sQ, sR + slot * HT_BYTES);
    mma_commit(&bars->s_full[t & 1]);
    mma_commit(&bars->free_[slot]);
  }
  mma_commit(&bars->scored);
}
__device__ void window_products(const Item& it, unsigned char* smem, Bars* bars, uint32_t tS, uint32_t tO) {
  const uint32_t sR = smem_u32(smem) + DA_OFF_RING;
  for (int t = 0; t < it.nt; ++t) {
    const int i = use_v(t, it.nt), slot = i % DA_NS;
    bool ok = needs_cleaning(it, it.t0 + t) ? mbar_wait_warp(&bars->clean[it.t0 + t - first_unclean(it)], 0u, &bars->abort)
                                            : mbar_wait_warp(&bars->full[slot], (uint32_t)(i / DA_NS) & 1u, &bars->abort);
    if (ok) ok = mbar_wait_warp(&bars->p_ready[t & 1], (uint32_t)(t >> 1) & 1u, &bars->abort);
    if (!ok) break;
    tc_fence_after();
    mma_weights(tO, tS + 64 * (t & 1), 32, sR + slot * HT_BYTES, t > 0, 4);
    mma_commit(&bars->pv_done[t & 1]);
    mma_commit(t + 1 < it.nt ? &bars->free_[slot] : &bars->o_full);      // (nothing follows into the last one's slot)
  }
}

// Returns how many uses have been asked for: all, unless a wait has run out (a slot whose last load may still be on its way is
// not armed again).
__device__ int window_load(const TcMaps& m, const Item& it, unsigned char* smem, Bars* bars) {
  for (int i = DA_NS; i < 2 * it.nt; ++i) {
    if (!mbar_wait_warp(&bars->free_[i % DA_NS], (uint32_t)(i / DA_NS - 1) & 1u, &bars->abort)) return i;
    load_use(m, it, smem, bars, i);
  }
  return 2 * it.nt;
}

__device__ void window_clean(const DraftArgs& d, const Item& it, unsigned char* smem, Bars* bars, int cid) {
  for (int T = first_unclean(it); T < it.t0 + it.nt; ++T) {
    const int n = T - first_unclean(it), slot = use_v(T - it.t0, it.nt) % DA_NS;
    if (!mbar_wait_warp(&bars->landed[n], 0u, &bars->abort)) return;
    unsigned char* tile = smem + DA_OFF_RING + slot * HT_BYTES;
    if (T < it.n_ring) {
      for (int c = cid + (it.held & 63) * 16; c < 64 * 16; c += 32) *reinterpret_cast<uint4*>(tile + at_half(c >> 4, c & 15)) = make_uint4(0u, 0u, 0u, 0u);
    } else {
      const int n0 = 64 * (T - it.n_ring);
#pragma unroll 4
      for (int c = cid; c < 64 * 16; c += 32) {
        uint4* p = reinterpret_cast<uint4*>(tile + at_half(c >> 4, c & 15));
        const int j = n0 + (c >> 4);
        const uint4 x = *p;
        const bool live = bars->depth[j] >= 0, odd = not_finite(x.x) || not_finite(x.y) || not_finite(x.z) || not_finite(x.w);
        if (!live || odd) *p = make_uint4(0u, 0u, 0u, 0u);
        if (live && odd) atomicOr(&bars->bad[j >> 5], 1u << (j & 31));
      }
    }
    fence_proxy_async_smem();
    mbar_arrive(&bars->clean[n]);
  }
}

// ---------------------------------------------------------------------------------------------------------- kernel

template <bool CL>
__global__ void __launch_bounds__(DA_THREADS, CL ? 1 : 2)
draft_tc_kernel(const __grid_constant__ TcArgs a, const __grid_constant__ TcMaps maps) {
  extern __shared__ __align__(1024) unsigned char smem[];
  Bars* bars = reinterpret_cast<Bars*>(smem + DA_OFF_BARS);
  const DraftArgs& d = a.d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = d.group;
  const int CS = CL ? a.cluster : 1, rank = CL ? (int)(blockIdx.x % CS) : 0;
  if (tid == 0) {
    const int rows = min(a.rows_per_tile, G * d.N - (int)(blockIdx.x / CS) % a.row_tiles * a.rows_per_tile);
    for (int i = 0; i < DA_NS; ++i) {
      mbar_init(&bars->full[i], 1);
      mbar_init(&bars->free_[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&bars->s_full[i], 1);
      mbar_init(&bars->pv_done[i], 1);
      mbar_init(&bars->p_ready[i], (uint32_t)((rows + 31) & ~31));      // the warps that have rows
    }
    mbar_init(&bars->q_full, 128);
    for (int i = 0; i < 3; ++i) {
      mbar_init(&bars->landed[i], 1);
      mbar_init(&bars->clean[i], 32);
    }
    mbar_init(&bars->scored, 1);
    mbar_init(&bars->o_full, 1);
    mbar_init(&bars->done, 1);
    mbar_init(&bars->drain, 2);
    bars->abort = 0;
    for (int i = 0; i < kMaxNodes / 32; ++i) bars->bad[i] = 0u;
    bars->n_far_node = bars->deepest = 0;
    fence_mbar_init();
  }
  if (warp == 4) {
    tmem_alloc(&bars->tmem_base, 256);
    tmem_relinquish();
  }
  if (tid == 160) {
    prefetch_tensormap(&maps.k_ring);
    prefetch_tensormap(&maps.v_ring);
    prefetch_map(&maps.k);
    prefetch_map(&maps.v);
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // (behind the allocation of TMEM: a kernel that is set up under this one may want some, too)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tmem = bars->tmem_base, tS = tmem, tO = tmem + 128, tFar = tO + 96;     // tFar: scores, then weights of far keys
  asm volatile("griddepcontrol.wait;" ::: "memory");        // the inputs may come from the kernel before
  const Item it = make_item(a, rank);

  if (warp == 5) {
    for (int i = 0; i < DA_NS && i < 2 * it.nt; ++i) load_use(maps, it, smem, bars, i);
  } else if (warp >= 6) {                                    // the tree; the state on its way to L2
    for (int n = tid - 192; n < kMaxNodes; n += 64) {
      const int p = n < d.N ? d.parents[(size_t)it.b * d.N + n] : -2;
      bars->par[n] = (signed char)(p == -1 || (p >= 0 && p < n) ? p : -2);
    }
    named_sync(1, 64);
    int deepest = 0;
    for (int n = tid - 192; n < kMaxNodes; n += 64) {
      int e = 0, j = n;
      for (;;) {
        const int p = bars->par[j];
        if (p < 0) { e = p == -1 ? e : -1; break; }
        j = p;
        ++e;
      }
      bars->depth[n] = (signed char)e;
      deepest = max(deepest, e);
    }
    deepest = __reduce_max_sync(0xffffffffu, deepest);
    if (lane == 0) atomicMax(&bars->deepest, deepest);
    const char* S = reinterpret_cast<const char*>(d.state + (size_t)it.z * TILE * TILE) + (size_t)rank * (TILE / CS) * 512;
    for (int i = tid - 192; i < TILE / CS * 4; i += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(S + i * 128));
  } else if (warp < 4) {
    // Q rows into the swizzled tile (rows beyond the item's are zero), 16 bytes at a time; they are awaited below
    const int c = tid & 15;
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(d.q) + node_at(d, it.b, it.hk * G, d.H_q, 0) + 8 * c;
    const size_t head = d.layout == RATTN_LAYOUT_BHTD ? (size_t)d.N * TILE : TILE, step = d.layout == RATTN_LAYOUT_BHTD ? TILE : (size_t)d.H_q * TILE;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int r = (tid >> 4) + 8 * i, row = it.row0 + min(r, it.rows - 1), n = small_div(row, a.inv_group);
      copy16_async(smem_u32(smem + at_tile(r, c)), q + (row - n * G) * head + n * step, r < it.rows);
    }
  }
  __syncthreads();

  const int dmax = bars->deepest;
  const RingAge age(it.pos, d.w);

  // this thread's row (row warps)
  const int node = warp < 4 && tid < it.rows ? small_div(it.row0 + tid, a.inv_group) : -1;
  const int e = node >= 0 ? bars->depth[node] : -1;
  const uint32_t lanes = (uint32_t)((tid & 96) << 16);       // TMEM lane of the row
  uint64_t near0 = 0, near1 = 0, far0 = 0, far1 = 0;         // nodes 0 - 63, 64 - 127 of its path, up to w levels up and further
  int uses = 0;                                              // of the ring's slots, asked for (loader warp)
  float m_ref = -INFINITY, l = 0.f;
  float inv_phi = 1.f;                                       // of the row's feature map
  // the slots behind the window's last use, oldest first: 0 - 2 are free once the last scores have been formed
  auto spare_slot = [&](int i) { return (2 * it.nt + i) % DA_NS; };
  auto spare = [&](int i) { return smem + DA_OFF_RING + spare_slot(i) * HT_BYTES; };
  const int corner = max(0, min(dmax, d.w) - age.first);     // far slots: ranks first .. first + corner - 1

  // ---- pieces of the linear branch.  Spare slots: 0, 1 the remainders of phi(Q); 2 phi(K_far), then V_far; 3, 4 half of S (64
  // features), leading parts and remainders.
  const uint32_t sQ = smem_u32(smem);
  const int k0 = 8 * rank / CS, k1 = 8 * (rank + 1) / CS;    // this CTA's steps of 16 features
  const int h0 = k0 >> 2;                                    // the (first) half that they lie in
  const float* S = d.state + (size_t)it.z * TILE * TILE;
  // phi(Q), while the last products run: every score has been formed, and every slot but those of the last two V tiles is free.
  // Leading parts go over Q, without the normalisation (inv_phi of the row's thread), remainders to the first two spare slots.
  // All four row warps: a row's thread takes all 16 pieces of eight features, or, where one or two warps have rows, two or four
  // threads in different warps share them.  (Loops that run once per row stay rolled: unrolled, they take as long as their
  // instructions take to arrive.  One thread per row took 4.4k cycles.)
  auto map_q = [&]() {
    const int row_warps = (it.rows + 31) >> 5, share = row_warps == 1 ? 4 : row_warps == 2 ? 2 : 1;      // threads per row
    const int r = share == 1 ? tid : lane + 32 * (warp % row_warps), part = share == 1 ? 0 : warp / row_warps;
    if (share == 1 && 32 * warp >= it.rows) return;          // (whole warps: rows behind the last are zero and mapped along)
    mbar_wait(&bars->q_full, 0u, &bars->abort);
    if (it.nt > 0 && part > 0) mbar_wait(&bars->scored, 0u, &bars->abort);        // (the row's own thread has seen the last scores)
    const int n = 16 / share, c0 = part * n, sw = r & 7;
    unsigned char* row = smem + r * 128;
    // [2][4][32 or 64]: maxima and sums of the threads that share a row, where the rows behind the last would have their remainders
    float* ex = reinterpret_cast<float*>(spare(0) + 64 * 128);
    float mq = 0.f, sq = 0.f;
    if (d.phi == RATTN_PHI_SOFTMAX) {
      mq = -INFINITY;
#pragma unroll 2
      for (int c = c0; c < c0 + n; ++c) {
        const uint4 u = *reinterpret_cast<const uint4*>(row + (c >> 3) * HALF_BYTES + (((c & 7) ^ sw) << 4));
        const uint32_t w4[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) mq = fmaxf(mq, fmaxf(__uint_as_float(w4[i] << 16), __uint_as_float(w4[i] & 0xffff0000u)));
      }
      if (share > 1) ex[part * 64 + r] = mq;
    }
    if (share > 1) {
      __syncwarp();
      named_sync(3, 128);
      if (d.phi == RATTN_PHI_SOFTMAX)
        for (int i = 0; i < share; ++i) mq = fmaxf(mq, ex[i * 64 + r]);
    }
    mq *= LOG2E;
    unsigned char* lo_row = spare(0) + r * 128;
    const ptrdiff_t lo_step = spare(1) - spare(0);
#pragma unroll 2
    for (int c = c0; c < c0 + n; ++c) {
      const int at = ((c & 7) ^ sw) << 4;
      uint4* p16 = reinterpret_cast<uint4*>(row + (c >> 3) * HALF_BYTES + at);
      const uint4 u = *p16;
      const uint32_t w4[4] = {u.x, u.y, u.z, u.w};
      uint32_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float p = __uint_as_float(w4[i] << 16), q = __uint_as_float(w4[i] & 0xffff0000u);
        if (d.phi == RATTN_PHI_SOFTMAX) {
          p = ex2(p * LOG2E - mq);
          q = ex2(q * LOG2E - mq);
          sq += p + q;
        } else if (d.phi == RATTN_PHI_RELU) {
          p = fmaxf(p, 0.f);
          q = fmaxf(q, 0.f);
        }
        split2(p, q, &hi[i], &lo[i]);
      }
      *p16 = make_uint4(hi[0], hi[1], hi[2], hi[3]);
      *reinterpret_cast<uint4*>(lo_row + (c >> 3) * lo_step + at) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
    fence_proxy_async_smem();
    if (share > 1) {
      ex[256 + part * 64 + r] = sq;
      __syncwarp();
      named_sync(3, 128);
      sq = 0.f;
      for (int i = 0; i < share; ++i) sq += ex[256 + i * 64 + r];
    }
    if (d.phi == RATTN_PHI_SOFTMAX) inv_phi = 1.f / sq;
  };
  // Half of S (128 threads, 16 float4 each), split, to the last two spare slots.  A CTA of many loads its second half and keeps it
  // while the first is multiplied; in a cluster there is one half, of which each CTA has a part, and eight loads at a time are
  // the smaller code (a chain of 6 for one sequence, inputs in L2: 12.9 against 13.6 us; elsewhere 4 % slower).
  constexpr int S_AHEAD = CL ? 8 : 16;
  float4 x_s[S_AHEAD];
  auto load_s = [&](int hh, int i0) {
    const int c = tid - 128;
#pragma unroll
    for (int i = 0; i < S_AHEAD; ++i) {
      const int f = 64 * hh + (c >> 5) + 4 * (i0 + i);
      x_s[i] = f >= 16 * k0 && f < 16 * k1 ? *reinterpret_cast<const float4*>(S + (size_t)f * TILE + (c & 31) * 4) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
  };
  auto store_s = [&](int i0) {
    const int c = tid - 128;
#pragma unroll
    for (int i = 0; i < S_AHEAD; ++i) {
      uint2 hi, lo;
      split2(x_s[i].x, x_s[i].y, &hi.x, &lo.x);
      split2(x_s[i].z, x_s[i].w, &hi.y, &lo.y);
      const uint32_t at = at_half((c >> 5) + 4 * (i0 + i), (c & 31) >> 1) + (c & 1) * 8;
      *reinterpret_cast<uint2*>(spare(3) + at) = hi;
      *reinterpret_cast<uint2*>(spare(4) + at) = lo;
    }
  };
  // products of the features 64 hh .. 64 hh + 63 with this CTA's part of S (MMA warp)
  auto mma_state = [&](int hh, bool acc) {
    constexpr uint32_t idesc = instr_desc(128, 128, 0, 1);
#pragma unroll
    for (int term = 0; term < 3; ++term) {                   // phi hi S hi, phi hi S lo, phi lo S hi
      const uint64_t a0 = kmajor_base(term == 2 ? smem_u32(spare(hh)) : sQ + hh * HALF_BYTES), b0 = mnmajor_base_h(smem_u32(spare(term == 1 ? 4 : 3)));
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (4 * hh + k >= k0 && 4 * hh + k < k1) {
          mma_bf16(tS, a0 + kstep_k(k, HALF_BYTES), b0 + kstep_mn(k), idesc, acc ? 1u : 0u);
          acc = true;
        }
    }
    return acc;
  };

  // phi(k) of far keys chunk .. chunk + 31 to the third spare slot, leading parts to its rows 0 - 31 and remainders to 32 - 63 (a row whose
  // linear branch is a handful of these shows their rounding: 2^-9 of a weight is as much as the output's own): a warp per
  // key, lane with 4 features
  auto far_source = [&](int i, bool is_v) -> const __nv_bfloat16* {
    if (i < corner) return static_cast<const __nv_bfloat16*>(is_v ? d.v_ring : d.k_ring) + ((size_t)it.z * d.w + age.slot(age.first + i)) * TILE;
    return static_cast<const __nv_bfloat16*>(is_v ? d.v : d.k) + node_at(d, it.b, it.hk, d.H_kv, bars->far_node[i - corner]);
  };
  auto build_k = [&](int chunk, int n_far, int first_warp, int n_warps) {
#pragma unroll 1
    for (int i = warp - first_warp; i < FAR && chunk + i < n_far; i += n_warps) {
      const uint2 u = reinterpret_cast<const uint2*>(far_source(chunk + i, false))[lane];
      float x[4] = {__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16), __uint_as_float(u.y & 0xffff0000u)};
      if (d.phi == RATTN_PHI_SOFTMAX) {
        const float m = wmax(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])));
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) s += x[j] = ex2((x[j] - m) * LOG2E);
        const float inv = 1.f / wsum(s);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] *= inv;
      } else if (d.phi == RATTN_PHI_RELU) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = fmaxf(x[j], 0.f);
      }
      uint2 hi, lo;
      split2(x[0], x[1], &hi.x, &lo.x);
      split2(x[2], x[3], &hi.y, &lo.y);
      unsigned char* to = spare(2) + at_half(i, lane >> 1) + (lane & 1) * 8;
      *reinterpret_cast<uint2*>(to) = hi;
      *reinterpret_cast<uint2*>(to + FAR * 128) = lo;
    }
    fence_proxy_async_smem();
  };

  if (warp < 4) {
    if (e >= 0) {
      for (int j = node, up = min(e, d.w); up >= 0; j = bars->par[j], --up) (j < 64 ? near0 : near1) |= 1ull << (j & 63);
      if (e > d.w)
        for (int j = node, up = 0; j >= 0; j = bars->par[j], ++up)
          if (up > d.w) (j < 64 ? far0 : far1) |= 1ull << (j & 63);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    fence_proxy_async_smem();
    mbar_arrive(&bars->q_full);
    if (32 * warp < it.rows) {
      const int ee = max(e, 0);
      for (int t = 0; t < it.nt; ++t) {
        const int T = it.t0 + t;
        const uint32_t ts = tS + 64 * (t & 1) + lanes;
        uint64_t keep;
        bool all;
        if (T < it.n_ring) {
          // slot s is kept if s < held and its rank is e or more
          const int s0 = 64 * T, h = age.head - s0;
          auto kept = [&](int depth) { return below(it.held - s0) & (~below(h + depth) | (below(h) & ~below(h + depth - d.w))); };
          all = kept(dmax) == ~0ull;
          keep = all ? ~0ull : kept(ee);
        } else {
          keep = T > it.n_ring ? near1 : near0;
          all = false;
        }
        if (!mbar_wait_warp(&bars->s_full[t & 1], (uint32_t)(t >> 1) & 1u, &bars->abort)) break;
        tc_fence_after();
        float x[64];
        tmem_ld32(ts, reinterpret_cast<float(&)[32]>(x[0]));
        tmem_ld32(ts + 32, reinterpret_cast<float(&)[32]>(x[32]));
        tmem_wait_ld();
        if (!all) {
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            if (!((uint32_t)keep >> i & 1u)) x[i] = -INFINITY;
            if (!((uint32_t)(keep >> 32) >> i & 1u)) x[32 + i] = -INFINITY;
          }
        }
        float mx = fmaxf(max32(reinterpret_cast<float(&)[32]>(x[0])), max32(reinterpret_cast<float(&)[32]>(x[32])));
        mx *= a.scale_log2;                                  // scale > 0
        // lazy rescale: the reference maximum moves when the row's grew by more than 2^8
        if (__any_sync(0xffffffffu, mx > m_ref + 8.f || m_ref == -INFINITY)) {
          const float m_new = fmaxf(m_ref, mx);
          if (t > 0) {
            const float f = m_new == -INFINITY ? 1.f : ex2(m_ref - m_new);
            if (!mbar_wait_warp(&bars->pv_done[(t - 1) & 1], (uint32_t)((t - 1) >> 1) & 1u, &bars->abort)) break;
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < 8; ++c) {
              float o[16];
              tmem_ld16(tO + lanes + 16 * c, o);
              tmem_wait_ld();
              uint32_t ow[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) ow[i] = __float_as_uint(o[i] * f);
              tmem_st16(tO + lanes + 16 * c, ow);
            }
            l *= f;
          }
          m_ref = m_new;
        }
        const float ms = m_ref == -INFINITY ? 0.f : m_ref;
        float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
        const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), nm2 = make_float2(-ms, -ms);
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float2 y = __ffma2_rn(make_float2(x[32 * c + 2 * i], x[32 * c + 2 * i + 1]), sc2, nm2);
            const float2 p = make_float2(ex2(y.x), ex2(y.y));
            if (i & 1) sum1 = __fadd2_rn(sum1, p);
            else sum0 = __fadd2_rn(sum0, p);
            split2(p.x, p.y, &hi[i], &lo[i]);
          }
          tmem_st16(ts + 16 * c, hi);
          tmem_st16(ts + 32 + 16 * c, lo);
        }
        l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
        tmem_wait_st();
        tc_fence_before();
#ifdef RATTN_DEBUG_KNOBS
        if (!(a.debug_wait == 1 && t == 0 && tid == 0 && rank == CS - 1))             // an arrival that never comes
#endif
        mbar_arrive(&bars->p_ready[t & 1]);
      }
    }
    map_q();
    if (32 * warp < it.rows) {
      if (it.nt > 0) mbar_wait(&bars->o_full, 0u, &bars->abort);
      tc_fence_after();
      __syncwarp();
    }
  } else if (warp == 4) {
    window_products(it, smem, bars, tS, tO);
#ifdef RATTN_DEBUG_KNOBS
    if (a.debug_wait == 2 && rank == CS - 1) bars->abort = 1;     // as if one of its waits had run out
#endif
  } else {
    if (warp == 5) uses = window_load(maps, it, smem, bars);
    else if (warp == 6) window_clean(d, it, smem, bars, lane);
    else window_scores(it, smem, bars, tS);
    // nodes that some row has more than w levels up; the far keys, as soon as there is room for them
    if (dmax > d.w && tid == 192) {
      int n = 0;
      for (int j = 0; j < d.N; ++j)
        if (bars->depth[j] >= 0 && bars->depth[j] < dmax - d.w) bars->far_node[n++] = (short)j;
      bars->n_far_node = n;
    }
    __syncwarp();
    named_sync(1, 96);
    mbar_wait(&bars->scored, 0u, &bars->abort);
    __syncwarp();
    if (rank == 0) build_k(0, corner + bars->n_far_node, 5, 3);
    if (!CL) load_s(0, 0);
  }
  // The window's products are complete, its slots free, all nodes looked at -- or a wait has run out, and all threads go to the
  // end.
  const bool gave_up = __syncthreads_or(*(volatile int*)&bars->abort) != 0;
  tc_fence_after();

  if (!gave_up) {
  // ---- linear branch -----------------------------------------------------------------------------------------------
  unsigned char* slots = smem + DA_OFF_RING;
  float* stat = reinterpret_cast<float*>(smem + DA_OFF_STAT);
  const int n_far = rank == 0 ? corner + bars->n_far_node : 0;
  const bool row_warp = warp < 4 && 32 * warp < it.rows;
  auto steps_of = [&](int chunk) { return (min(FAR, n_far - chunk) + 15) >> 4; };
  // values of the far keys, zero behind the last and for nodes that are not finite: to registers (128 threads, a warp per key),
  // and over their keys
  auto load_v = [&](int chunk, uint2 (&u)[FAR / 4]) {
#pragma unroll
    for (int j = 0; j < FAR / 4; ++j) {
      const int i = chunk + warp - 4 + 4 * j;
      u[j] = make_uint2(0u, 0u);
      if (i < n_far) {
        u[j] = reinterpret_cast<const uint2*>(far_source(i, true))[lane];
        if (i >= corner && (not_finite(u[j].x) || not_finite(u[j].y))) u[j] = make_uint2(0u, 0u);
      }
    }
  };
  auto store_v = [&](const uint2 (&u)[FAR / 4]) {
#pragma unroll
    for (int j = 0; j < FAR / 4; ++j) *reinterpret_cast<uint2*>(spare(2) + at_half(warp - 4 + 4 * j, lane >> 1) + (lane & 1) * 8) = u[j];
    fence_proxy_async_smem();
  };
  // the scores of the far keys become weights: those of corner keys of rank below e and of nodes on the path more than w levels up
  auto far_weights = [&](int chunk) {
    uint32_t keep = (uint32_t)below(min(corner, max(e, 0) - age.first) - chunk);
    for (int i = max(corner - chunk, 0); i < FAR && chunk + i < n_far; ++i) {
      const int j = bars->far_node[chunk + i - corner];
      if ((j < 64 ? far0 : far1) >> (j & 63) & 1u) keep |= 1u << i;
    }
    float z[32];
    tmem_ld32(tFar + lanes, z);
    tmem_wait_ld();
    uint32_t hi[16], lo[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) split2(keep >> (2 * i) & 1u ? z[2 * i] : 0.f, keep >> (2 * i + 1) & 1u ? z[2 * i + 1] : 0.f, &hi[i], &lo[i]);
    tmem_st16(tFar + lanes, hi);
    tmem_st16(tFar + FAR / 2 + lanes, lo);
    tmem_wait_st();
  };
  auto mma_far_scores = [&](int chunk) {                      // phi(Q) phi(K_far)^T: hi hi, lo hi, hi lo
    const uint32_t idesc = instr_desc(128, 16 * steps_of(chunk), 0, 0);
#pragma unroll
    for (int term = 0; term < 3; ++term) {
      const uint64_t a0 = kmajor_base(term == 1 ? smem_u32(spare(0)) : sQ), a1 = kmajor_base(term == 1 ? smem_u32(spare(1)) : sQ + HALF_BYTES);
      const uint64_t b0 = kmajor_base_h(smem_u32(spare(2)) + (term == 2 ? FAR * 128 : 0));
#pragma unroll
      for (int k = 0; k < 8; ++k)
        mma_bf16(tFar, (k < 4 ? a0 : a1) + kstep_k(k & 3, HALF_BYTES), b0 + kstep_k(k, HT_HALF), idesc, (term > 0 || k > 0) ? 1u : 0u);
    }
  };

  // What the row in this thread's lane of an accumulator, `by` times it being a branch's output, is to be multiplied by: by / rms.
  // A sum of squares that overflows is formed again from values scaled down (row_inv_rms).
  auto norm_scale = [&](uint32_t at, float by) {
    float scale = by, down = 1.f;
#pragma unroll 1
    for (;;) {
      float ss = 0.f;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        float o[32];
        tmem_ld32(at + lanes + 32 * c, o);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 32; ++i) ss += (o[i] * scale) * (o[i] * scale);
      }
      const float f = scale * rsqrtf(ss * (1.f / TILE) + d.eps * down * down);
      const bool again = down == 1.f && ss == INFINITY;
      if (!__any_sync(0xffffffffu, again)) return f;
      // (rows that stay as they are keep their scale and are summed along)
      if (again) {
        down = kDown;
        scale = by * kDown;
      }
    }
  };

  uint2 v_far[FAR / 4];
  float window_scale = 0.f;                                  // one-CTA path: of this thread's row
  if (row_warp) {
    // the window output leaves the accumulator
    const uint64_t bad0 = (uint64_t)bars->bad[1] << 32 | bars->bad[0], bad1 = (uint64_t)bars->bad[3] << 32 | bars->bad[2];
    const bool seen = (((near0 | far0) & bad0) | ((near1 | far1) & bad1)) != 0;
    if (CL) {
      if (tid < DA_CLUSTER_ROWS) {
        stat[tid] = m_ref;
        stat[DA_CLUSTER_ROWS + tid] = seen ? __uint_as_float(0x7fc00000u) : l;
      }
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        float o[32];
        if (it.nt > 0) {
          tmem_ld32(tO + lanes + 32 * c, o);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = 0.f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<float4*>(smem + DA_OFF_OX + at_ox(tid, 8 * c + i)) = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
      }
    } else {
      const float inv = (seen ? __uint_as_float(0x7fc00000u) : 1.f) / l;
      window_scale = norm_scale(tO, inv);
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        float o[32];
        tmem_ld32(tO + lanes + 32 * c, o);
        tmem_wait_ld();
        uint32_t a16[16], a8[8];                             // 24 words over columns that have been read
#pragma unroll
        for (int i = 0; i < 8; ++i) pack24(o + 4 * i, &a16[2 * i], &a16[2 * i + 1], &a8[i]);
        tmem_st16(tO + lanes + 24 * c, a16);
        tmem_st8(tO + lanes + 24 * c + 16, a8);
      }
      tmem_wait_st();
    }
  }

  else if (warp >= 4) {
    // phi(Q) S meanwhile, half of the features after the other
    if (!CL && warp == 4) load_s(0, 0);
    bool acc = false;
#pragma unroll 1
    for (int hh = h0; hh < 2; ++hh) {
      if (hh > h0) {
        if (CL) break;                                       // (the CTAs of a cluster have features of one half each)
        mbar_wait(&bars->done, 0u, &bars->abort);
        __syncwarp();
      }
      if (CL) {
#pragma unroll 1
        for (int i0 = 0; i0 < 16; i0 += S_AHEAD) {
          load_s(hh, i0);
          store_s(i0);
        }
      } else {
        store_s(0);
      }
      fence_proxy_async_smem();
      if (!CL && hh == 0) load_s(1, 0);
      named_sync(2, 128);
      if (warp == 4) {
        tc_fence_after();
        acc = mma_state(hh, acc);
        if (!CL && hh == 0) mma_commit(&bars->done);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  // Far keys, 32 at a time (the first of them are mapped already).  The first commit also covers the products above.  (One copy of
  // this code, whatever their number: what a CTA executes once it has to wait for.)
  uint32_t done_phase = CL ? 0 : 1;
  auto wait_done = [&]() {
    mbar_wait(&bars->done, done_phase++ & 1u, &bars->abort);
    __syncwarp();
    tc_fence_after();
  };
  int chunk = 0;
#pragma unroll 1
  do {
    if (chunk > 0) {
      if (warp >= 4) build_k(chunk, n_far, 4, 4);
      tc_fence_before();
      __syncthreads();
      tc_fence_after();
    }
    if (warp == 4) {
      if (n_far > 0) mma_far_scores(chunk);
      mma_commit(&bars->done);
    }
    if (warp >= 4) load_v(chunk, v_far);
    wait_done();
    if (n_far == 0) break;                                   // (the same for all threads)
    if (warp >= 4) store_v(v_far);
    else if (row_warp) far_weights(chunk);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 4) {
      mma_weights(tS, tFar, FAR / 2, smem_u32(spare(2)), true, steps_of(chunk));
      mma_commit(&bars->done);
    }
    wait_done();
    chunk += FAR;
  } while (chunk < n_far);

  // ---- Section 3.2: two RMS norms and the sum ------------------------------------------------------------------------
  if (CL) {
    if (row_warp) {
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        float o[32];
        tmem_ld32(tS + lanes + 32 * c, o);
        tmem_wait_ld();
#pragma unroll
        for (int i = 0; i < 8; ++i)
          *reinterpret_cast<float4*>(smem + DA_OFF_OX + DA_CLUSTER_ROWS * 512 + at_ox(tid, 8 * c + i)) =
              make_float4(o[4 * i] * inv_phi, o[4 * i + 1] * inv_phi, o[4 * i + 2] * inv_phi, o[4 * i + 3] * inv_phi);
      }
      tc_fence_before();
    }
    __syncthreads();
    const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
    const int c0 = 4 * lane;
    float4 gs = one, gr = one;
    auto gains = [&](int r) {
      if (r >= it.rows) return;
      const int n = small_div(it.row0 + r, a.inv_group);
      const size_t at = (size_t)(it.hk * G + it.row0 + r - n * G) * TILE + c0;
      if (d.gamma_swa) gs = *reinterpret_cast<const float4*>(d.gamma_swa + at);
      if (d.gamma_rla) gr = *reinterpret_cast<const float4*>(d.gamma_rla + at);
    };
    gains(rank + CS * warp);                                 // (on their way while the cluster meets)
    cluster_arrive();                                        // partial outputs of every CTA are in place
    cluster_wait();
    // a wait that ran out in one of the CTAs ends the call for all of them
    const bool ok = !__any_sync(0xffffffffu, lane < CS && __float_as_uint(ld_cluster(cluster_addr(&bars->abort, lane))) != 0u);
    for (int r = rank + CS * warp; ok && r < it.rows; r += CS * (DA_THREADS / 32)) {
      const int n = small_div(it.row0 + r, a.inv_group), h = it.hk * G + it.row0 + r - n * G;
      if (r >= CS * (DA_THREADS / 32)) gains(r);
      if (bars->depth[n] < 0) continue;
      float4 p[8], q[8];
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < CS) {
          p[k] = ld_cluster4(cluster_addr(smem + DA_OFF_OX + at_ox(r, lane), k));
          q[k] = ld_cluster4(cluster_addr(smem + DA_OFF_OX + DA_CLUSTER_ROWS * 512 + at_ox(r, lane), k));
        }
      float m_r = -INFINITY, l_r = 0.f;
      if (lane < CS) {
        m_r = ld_cluster(cluster_addr(stat + r, lane));
        l_r = ld_cluster(cluster_addr(stat + DA_CLUSTER_ROWS + r, lane));
      }
      const float m = wmax(m_r), f = ex2(m_r - (m == -INFINITY ? 0.f : m));
      const float inv = 1.f / wsum(lane < CS ? f * l_r : 0.f);
      float x[4] = {0.f, 0.f, 0.f, 0.f}, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (k < CS) {
          const float fr = __shfl_sync(0xffffffffu, f, k) * inv;
          x[0] += fr * p[k].x; x[1] += fr * p[k].y; x[2] += fr * p[k].z; x[3] += fr * p[k].w;
          y[0] += q[k].x; y[1] += q[k].y; y[2] += q[k].z; y[3] += q[k].w;
        }
      const float is = row_inv_rms(x, d.eps), ir = row_inv_rms(y, d.eps);
      *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(d.out) + node_at(d, it.b, h, d.H_q, n) + c0) =
          make_uint2(pack_bf16(gs.x * x[0] * is + gr.x * y[0] * ir, gs.y * x[1] * is + gr.y * y[1] * ir),
                     pack_bf16(gs.z * x[2] * is + gr.z * y[2] * ir, gs.w * x[3] * is + gr.w * y[3] * ir));
    }
  } else {
   auto at_row = [&](int r, int c) { return (uint32_t)(r * 256 + ((c ^ (r & 15)) << 4)); };
   auto at_third = [&](int r, int c) { return (uint32_t)(r * 128 + ((c ^ (r & 7)) << 4)); };
   if (row_warp) {
    const float f = norm_scale(tS, inv_phi);
    // the window branch as it was packed, two words of each three in rows of 256 bytes over Q, the third in rows of 128 over slot 4; the
    // linear one, normalised, fp32 rows over slots 0 - 3
    bars->window_scale[tid] = window_scale;                  // (nobody looks for parents or far nodes any more)
#pragma unroll 1
    for (int c = 0; c < 4; ++c) {
      float o[32], s16[16], s8[8];
      tmem_ld32(tS + lanes + 32 * c, o);
      tmem_ld16(tO + lanes + 24 * c, s16);
      tmem_ld8(tO + lanes + 24 * c + 16, s8);
      tmem_wait_ld();
#pragma unroll
      for (int i = 0; i < 2; ++i)
        *reinterpret_cast<float4*>(slots + 4 * HT_BYTES + at_third(tid, 2 * c + i)) = make_float4(s8[4 * i], s8[4 * i + 1], s8[4 * i + 2], s8[4 * i + 3]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<uint4*>(smem + at_row(tid, 4 * c + i)) =
            make_uint4(__float_as_uint(s16[4 * i]), __float_as_uint(s16[4 * i + 1]), __float_as_uint(s16[4 * i + 2]), __float_as_uint(s16[4 * i + 3]));
#pragma unroll
      for (int i = 0; i < 8; ++i)
        *reinterpret_cast<float4*>(slots + at_ox(tid, 8 * c + i)) = make_float4(o[4 * i] * f, o[4 * i + 1] * f, o[4 * i + 2] * f, o[4 * i + 3] * f);
    }
    tc_fence_before();
   }
   __syncthreads();
   if (!*(volatile int*)&bars->abort) {
    // Head by head, so that its gains are read once; a warp takes every eighth of a head's rows, which are G apart.
    const int c0 = 4 * lane, n0 = small_div(it.row0, a.inv_group), g0 = it.row0 - n0 * G;
    const float4 one = make_float4(1.f, 1.f, 1.f, 1.f);
    auto gain_of = [&](const float* gamma, int i) {
      const int g = g0 + i, h = it.hk * G + (g >= G ? g - G : g);
      return gamma && i < G ? *reinterpret_cast<const float4*>(gamma + (size_t)h * TILE + c0) : one;
    };
    float4 gs = gain_of(d.gamma_swa, 0), gr = gain_of(d.gamma_rla, 0);
    const size_t step = (d.layout == RATTN_LAYOUT_BHTD ? (size_t)TILE : (size_t)d.H_q * TILE) * (DA_THREADS / 32);
#pragma unroll 1
    for (int i = 0; i < G && i < it.rows; ++i) {             // rows i, i + G, ..: head g of nodes n, n + 1, ..
      const float4 gs_next = gain_of(d.gamma_swa, i + 1), gr_next = gain_of(d.gamma_rla, i + 1);
      const int wrap = g0 + i >= G, h = it.hk * G + g0 + i - (wrap ? G : 0);
      // (heads in turn start with another warp, so that few rows are shared out)
      const int k0_ = (warp - i) & 7;
      __nv_bfloat16* out = static_cast<__nv_bfloat16*>(d.out) + node_at(d, it.b, h, d.H_q, n0 + wrap + k0_) + c0;
#pragma unroll 2
      for (int k = k0_; i + G * k < it.rows; k += DA_THREADS / 32, out += step) {
        const int r = i + G * k;
        if (bars->depth[n0 + wrap + k] < 0) continue;
        const uint2 u = *reinterpret_cast<const uint2*>(smem + at_row(r, lane >> 1) + (lane & 1) * 8);
        const uint32_t u2 = *reinterpret_cast<const uint32_t*>(slots + 4 * HT_BYTES + at_third(r, lane >> 2) + (lane & 3) * 4);
        const float4 y = *reinterpret_cast<const float4*>(slots + at_ox(r, lane)), x = unpack24(u.x, u.y, u2);
        const float f = bars->window_scale[r];
        *reinterpret_cast<uint2*>(out) =
            make_uint2(pack_bf16(gs.x * (x.x * f) + gr.x * y.x, gs.y * (x.y * f) + gr.y * y.y),
                       pack_bf16(gs.z * (x.z * f) + gr.z * y.z, gs.w * (x.w * f) + gr.w * y.w));
      }
      gs = gs_next;
      gr = gr_next;
    }
   }
  }
  } else if (CL) {                                           // (the others learn of it behind this barrier)
    cluster_arrive();
    cluster_wait();
  }
  if (*(volatile int*)&bars->abort) {
    // a wait ran out: what is still in flight gets a bounded time to land before the memory goes away
    if (warp == 7) mma_commit(&bars->drain);
    if (warp == 4) {
      mma_commit(&bars->drain);
      for (int i = 0; i < kWaitPolls && !mbar_try_wait(&bars->drain, 0u); ++i) {}
    }
    if (warp == 5) {
      for (int i = max(0, uses - DA_NS); i < uses; ++i)
        for (int p = 0; p < kWaitPolls && !mbar_try_wait(&bars->full[i % DA_NS], (uint32_t)(i / DA_NS) & 1u); ++p) {}
      for (int T = first_unclean(it); T < it.t0 + it.nt && use_v(T - it.t0, it.nt) < uses; ++T)
        for (int p = 0; p < kWaitPolls && !mbar_try_wait(&bars->landed[T - first_unclean(it)], 0u); ++p) {}
    }
    if (tid == 0) g_draft_status = RATTN_ERR_TIMEOUT;
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (warp == 4) {
    tc_fence_after();
    tmem_dealloc(tmem, 256);
  }
  if (CL) {                                                  // nobody leaves while its outputs are being read
    __syncwarp();
    cluster_arrive();
    cluster_wait();
  }
}

template <bool CL>
cudaError_t launch(const TcArgs& a, const TcMaps& m, int items, cudaStream_t s) {
  constexpr int smem = CL ? DA_SMEM_CLUSTER : DA_SMEM;
  cudaError_t e = allow_smem<draft_tc_kernel<CL>>(smem);
  if (e != cudaSuccess) return e;
  {
    KernelTimer kt("draft_attention", s);
    e = launch_pdl_cluster(draft_tc_kernel<CL>, dim3((unsigned)(items * a.cluster)), dim3(DA_THREADS), smem, s, true, a.cluster, a, m);
    if (e != cudaSuccess) return e;
  }
  count_launches(1);
  return cudaGetLastError();
}

}  // namespace

bool tc_applies(const DraftArgs& a) {
  return a.dtype == RATTN_BF16 && a.d == TILE && a.scale > 0.f && a.group <= 4096 && !(a.flags & RATTN_FLAG_FORCE_GENERIC);
}

cudaError_t launch_tc(const DraftArgs& d, cudaStream_t s) {
  TcArgs a;
  TcMaps m;
  a.d = d;
  a.scale_log2 = d.scale * LOG2E;
  a.inv_group = 1.f / (float)d.group;
  a.debug_wait = debug_wait();
  if (!make_map(&m.k_ring, d.k_ring, (uint64_t)d.w, (uint64_t)d.B * d.H_kv, 64) ||
      !make_map(&m.v_ring, d.v_ring, (uint64_t)d.w, (uint64_t)d.B * d.H_kv, 64) ||
      !make_user_map(&m.k, d.k, (uint64_t)d.N, (uint64_t)d.H_kv, (uint64_t)d.B, d.layout, 64) ||
      !make_user_map(&m.v, d.v, (uint64_t)d.N, (uint64_t)d.H_kv, (uint64_t)d.B, d.layout, 64))
    return cudaErrorInvalidValue;
  const long long R = (long long)d.group * d.N, heads = (long long)d.B * d.H_kv;
  const int tiles = ((d.pos_dev || d.pos >= d.w ? d.w : d.pos) + 63) / 64 + (d.N + 63) / 64;
  // Row tiles of a cluster hold at most 96 rows (what the exchange has room for); a cluster has as many CTAs as let all clusters run
  // at once, and no more than there are tiles of keys (4 query heads x 6 nodes per K/V head, w = 512; CTAs per cluster 1 / 2 / 4 / 8:
  // 15 heads 22.0 / 16.8 / 14.7 / 14.0 us, 16 heads 22.1 / 16.9 / 14.4 / 25.8 where 15 clusters of eight run at once; 33 of four: 36
  // heads 23.1 / 17.2 / 28.6; 74 of two: 74 heads 21.2 / 19.0, 75 heads 22.9).
  const long long rt_c = (R + DA_CLUSTER_ROWS - 1) / DA_CLUSTER_ROWS;
  int cs = 1, fit = 0;
  cudaError_t e = allow_smem<draft_tc_kernel<true>>(DA_SMEM_CLUSTER);
  while (e == cudaSuccess && cs < 8 && 2 * cs <= tiles) {
    e = clusters_at_once<draft_tc_kernel<true>>(2 * cs, DA_THREADS, DA_SMEM_CLUSTER, &fit);
    if (heads * rt_c > fit) break;
    cs *= 2;
  }
  if (e != cudaSuccess) return e;
  a.cluster = cs;
  a.row_tiles = (int)(cs > 1 ? rt_c : (R + TILE - 1) / TILE);
  a.rows_per_tile = (int)((R + a.row_tiles - 1) / a.row_tiles);
  a.row_tiles = (int)((R + a.rows_per_tile - 1) / a.rows_per_tile);
  const long long items = heads * a.row_tiles;
  return cs > 1 ? launch<true>(a, m, (int)items, s) : launch<false>(a, m, (int)items, s);
}

int tc_status(cudaStream_t s, cudaError_t* err) {
  int word = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(&word, g_draft_status, sizeof(int), 0, cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e == cudaSuccess && word != 0) {
    const int zero = 0;
    e = cudaMemcpyToSymbolAsync(g_draft_status, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  }
  *err = e;
  return word;
}

}  // namespace draft
}  // namespace rattn
