// Attention of a tree of drafted tokens over paged, un-rotated K/V (§3.3.3): what its kernels share. Row i of request b (a node and a
// query head) computes
//   out_i = sum_n w_in v_n / sum_n w_in,   w_in = 2^(s_in - m_i),   s_in = scale log2(e) (R(p_i) q_i) . (R(p(n)) k_n)
// over the context slots n < C (all valid ones) and the nodes on the path from the root to its own, node j being slot C + j.
#pragma once
#include "attn_scalar.h"

namespace mepic {

constexpr int kTreeWords = MEPIC_TREE_MAX_NODES / 32;  // words of a node's path

struct TreeArgs {
  AttnArgs a;              // cu_q_lens set; causal unused
  const int32_t* parents;  // null: chains
  int32_t max_q;           // host's bound on nodes per request, at most MEPIC_TREE_MAX_NODES
};

// One request as the kernels see it.
struct TreeRequest {
  int q0, T;   // first query token, nodes
  int kv_len;  // slots, nodes included, forced into the table
  int ctx;     // slot of node 0 (negative where there are fewer slots than nodes)
};

__device__ __forceinline__ TreeRequest tree_request(const AttnArgs& a, int b) {
  TreeRequest r;
  r.q0 = min(max(a.cu_q_lens[b], 0), a.n_q);  // (nothing on the device is taken on trust where it forms an address)
  r.T = min(max(a.cu_q_lens[b + 1] - r.q0, 0), a.n_q - r.q0);
  r.kv_len = max(min(a.kv_lens[b], a.max_blocks * a.P), 0);
  r.ctx = r.kv_len - r.T;
  return r;
}

// The parent of node j, -1 for a root.
__device__ __forceinline__ int tree_parent(const int32_t* parents, int q0, int j) {
  const int p = parents ? parents[q0 + j] : j - 1;
  return p >= 0 && p < j ? p : -1;
}

// The low n bits, n from anything below 0 to anything above 32.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1u; }

// Bits of slots n0 .. n0 + 31 that a row sees: all of the context's, of the nodes those on its path.
__device__ __forceinline__ uint32_t path_bits(const uint32_t* path, int n0, int ctx) {
  const int off = n0 - ctx;  // bit i is node off + i
  if (off <= -32) return ~0u;
  if (off < 0) return low_bits(-off) | (path[0] << -off);
  const int w = off >> 5, s = off & 31;
  const uint32_t lo = w < kTreeWords ? path[w] >> s : 0u;
  return s && w + 1 < kTreeWords ? lo | (path[w + 1] << (32 - s)) : lo;
}

template <int kThreads>
struct TreeRowLds {
  float qhat[2 * kMaxHalfD];  // rotated, times scale log2(e)
  float w[kThreads];          // weights of a tile's slots
  float red[kThreads / 64];
  uint32_t path[kTreeWords];
};

// Load one 16-byte granule and widen it to fp32 (e4m3 NaN codes are NaN).
template <int KV>
__device__ __forceinline__ void tree_granule(const void* base, size_t granule_index, float* x) {
  if constexpr (KV == MEPIC_F8E4M3) {
    const uint4 g = reinterpret_cast<const uint4*>(base)[granule_index];
    const uint32_t u[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8(u[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8(u[i], true);
      x[4 * i] = lo[0]; x[4 * i + 1] = lo[1]; x[4 * i + 2] = hi[0]; x[4 * i + 3] = hi[1];
    }
  } else {
    load_granule<KV>(base, granule_index, x);
  }
}

// One output row (query token t = node `node` of request b, query head hq) in plain fp32 arithmetic, by all threads of the workgroup.
// A slot the row does not see is not multiplied, whatever it holds. A thread has a slot of a tile of kThreads for the scores, then a
// dim (one of kThreads / D threads each) for the sum over V.
template <int KV, int kThreads>
__device__ __forceinline__ void tree_row(const TreeArgs& ta, TreeRowLds<kThreads>& lds, const TreeRequest& r, int b, int node, int hq) {
  constexpr int X = Store<KV>::X, kWaves = kThreads / 64;
  using T = typename Store<KV>::T;
  const AttnArgs& a = ta.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int D = a.D, P = a.P, half = D / 2, hk = hq / a.G;
  const size_t row = ((size_t)(r.q0 + node) * a.Hq + hq) * D;
  __syncthreads();  // (the last row's reads of lds)
  if (tid < half) {
    const int i0 = a.interleaved ? 2 * tid : tid, i1 = a.interleaved ? 2 * tid + 1 : tid + half;
    const float x0 = load_q(a.q, a.q_dtype, row + i0), x1 = load_q(a.q, a.q_dtype, row + i1);
    float sn, cs;
    sincospif(2.0f * turns_frac((float)a.q_positions[r.q0 + node], a.freq_hi[tid], a.freq_lo[tid]), &sn, &cs);
    lds.qhat[i0] = (x0 * cs - x1 * sn) * a.qk_scale_log2;
    lds.qhat[i1] = (x1 * cs + x0 * sn) * a.qk_scale_log2;
  }
  if (tid == 0) {
    uint32_t path[kTreeWords] = {};
    for (int j = node, steps = 0; j >= 0 && steps < MEPIC_TREE_MAX_NODES; j = tree_parent(ta.parents, r.q0, j), ++steps)
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w) path[w] |= (j >> 5) == w ? 1u << (j & 31) : 0u;
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) lds.path[w] = path[w];
  }
  __syncthreads();

  const int d_own = tid % D, part = tid / D, parts = kThreads / D;
  float acc = 0.f, m = -INFINITY, l = 0.f;
  const size_t bt_row = (size_t)b * a.max_blocks;
  const float* q = lds.qhat;
  for (int n0 = 0; n0 < r.kv_len; n0 += kThreads) {
    const int n = n0 + tid, j = n - r.ctx;
    bool take = n < r.kv_len && (j < 0 || ((lds.path[(j >> 5) & (kTreeWords - 1)] >> (j & 31)) & 1u));
    if (j >= MEPIC_TREE_MAX_NODES) take = false;
    if (take && a.block_valid_mask) take = (a.block_valid_mask[bt_row + n / P] >> (n % P)) & 1u;
    float s = -INFINITY;
    if (take) {
      const int page = max(min(a.block_tables[bt_row + n / P], a.num_pages - 1), 0), sl = n % P;
      int pos = n;
      if (j >= 0) pos = a.q_positions[r.q0 + j];
      else if (a.block_positions) pos = a.block_positions[bt_row + n / P] + sl;
      const size_t granules = ((size_t)page * a.Hkv + hk) * (size_t)(D / X) * P;
      const int step = a.interleaved ? 1 : 2;  // granules that hold whole pairs
      const int pairs = X * step / 2;          // pairs in them
      float dot = 0.f;
      for (int c = 0; c < D / X / step; ++c) {
        float x0[X], x1[X];
        tree_granule<KV>(a.k_pages, granules + (size_t)c * P + sl, x0);
        if (!a.interleaved) tree_granule<KV>(a.k_pages, granules + (size_t)(c + D / X / 2) * P + sl, x1);
#pragma unroll
        for (int e = 0; e < X; ++e) {
          if (e < pairs) {
            const int i = c * pairs + e;
            float sn, cs;
            sincospif(2.0f * turns_frac((float)pos, a.freq_hi[i], a.freq_lo[i]), &sn, &cs);
            const float lo = a.interleaved ? x0[(2 * e) % X] : x0[e], hi = a.interleaved ? x0[(2 * e + 1) % X] : x1[e];
            const float qlo = a.interleaved ? q[2 * i] : q[i], qhi = a.interleaved ? q[2 * i + 1] : q[i + half];
            dot += qlo * (lo * cs - hi * sn) + qhi * (hi * cs + lo * sn);
          }
        }
      }
      s = KV == MEPIC_F8E4M3 ? dot * a.k_scales[page] : dot;
    }
    const float wm = wave_max(s);
    if (lane == 0) lds.red[wave] = wm;
    __syncthreads();
    float m_new = m;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m_new = fmaxf(m_new, lds.red[w]);
    const float f = m_new == -INFINITY ? 1.f : exp2f(m - m_new);
    m = m_new;
    const float w = take ? exp2f(s - (m == -INFINITY ? 0.f : m)) : 0.f;
    lds.w[tid] = take ? w : -1.f;  // (a weight is never negative; it may be NaN)
    __syncthreads();  // (red is read)
    const float ws = wave_sum(w);
    if (lane == 0) lds.red[wave] = ws;
    __syncthreads();
    l *= f;
    acc *= f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) l += lds.red[i];
    const int blocks = (min(kThreads, r.kv_len - n0) + P - 1) / P;  // n0 is a multiple of P
    for (int jb = part; jb < blocks; jb += parts) {
      const int page = max(min(a.block_tables[bt_row + (n0 + jb * P) / P], a.num_pages - 1), 0);
      const float vs = KV == MEPIC_F8E4M3 ? a.v_scales[page] : 1.f;
      const T* v = reinterpret_cast<const T*>(a.v_pages) + (((size_t)page * a.Hkv + hk) * D + d_own) * (size_t)P;
      for (int c = 0; c < P / X; ++c) {
        float x[X];
        tree_granule<KV>(v, c, x);
#pragma unroll
        for (int e = 0; e < X; ++e) {
          const float we = lds.w[jb * P + c * X + e];
          if (!(we < 0.f)) acc += we * (x[e] * vs);
        }
      }
    }
    __syncthreads();  // (w and red are written anew)
  }
  lds.w[tid] = acc;
  __syncthreads();
  if (part == 0) {
    float o = 0.f;
    for (int p = 0; p < parts; ++p) o += lds.w[p * D + d_own];
    const float x = l != 0.f ? o / l : 0.f;
    if (a.q_dtype == MEPIC_F32) reinterpret_cast<float*>(a.out)[row + d_own] = x;
    else reinterpret_cast<uint16_t*>(a.out)[row + d_own] = (uint16_t)pack2_bf16(x, x);
  }
}

// The request that owns query token t, or -1 for a row behind the last one (the prefix sums ascend; empty requests own nothing).
__device__ __forceinline__ int request_of(const int32_t* cu, int B, int t) {
  if (t >= cu[B] || t < cu[0]) return -1;
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= t) lo = mid; else hi = mid;
  }
  return lo;
}

// How a call of the matrix-core kernels is cut (tree_mfma_plan).
struct TreePlan {
  int rows;        // rows of a workgroup's tile: 32, 64, 128, 256
  int groups;      // workgroups per KV head
  int min_slots;   // least run of a workgroup
  bool whole;      // a workgroup takes whole items (row tiles of a request): nothing to merge
  int row_tiles, splits;  // fp32 pages: row tiles per request, workgroups per item
  size_t bytes;    // workspace
};

struct TreeMfmaArgs {
  TreeArgs t;
  int32_t groups, min_slots, whole;
  float* part_o;     // [groups * Hkv][2][rows][D]
  float* part_ml;    // [groups * Hkv][2][rows][2]
  int4* row_wgs;     // [n_q * G] first and last workgroup (of a KV head) that a row's item is cut for, row of the tile, request
};

struct TreeF32Args {
  TreeArgs t;
  int32_t row_tiles, splits;
  float* part_o;   // [B * row_tiles][splits][Hkv][16][D]
  float* part_ml;  // [B * row_tiles][splits][Hkv][16][2]
};

TreePlan tree_f32_plan(const TreeArgs& t, int max_kv);
hipError_t launch_tree_f32(const TreeArgs& t, const TreePlan& pl, void* workspace, hipStream_t s);
TreePlan tree_mfma_plan(const TreeArgs& t, int max_kv);  // reads shapes and max_q; rows = 0: the general kernel's
hipError_t launch_tree_mfma(const TreeArgs& t, const TreePlan& pl, void* workspace, hipStream_t s);  // bf16 or e4m3 pages; with its merge and timing_stop
hipError_t launch_tree_tiles_bf16(int rows, const TreeMfmaArgs& m, hipStream_t s);
hipError_t launch_tree_tiles_fp8(int rows, const TreeMfmaArgs& m, hipStream_t s);
hipError_t launch_tree_general(const TreeArgs& t, hipStream_t s);  // any form, plain fp32 arithmetic

}  // namespace mepic
