// Attention of a tree of drafted tokens on the matrix cores, fp32 pages: the formula of tree_common.h with fp32 operands throughout.
//
// v_mfma_f32_16x16x4_f32 bounds it (2 x 32 of them, 32 clocks each, for 16 slots x 16 rows of D 128), so nothing goes through LDS in the loop:
// a wave takes 16 rows of a request and 16 slots a step, and both operands come from memory in operand order. Contractions may run in any
// order: lane (n, g) of a step holds of slot n the granules 4 i + g (whole rotary pairs), and element e of granule i is one product's operand
// next to the same elements of Q; of V it holds for dim 16 dt + n the slots 4 g .. 4 g + 3, whose weights the scores' product has left
// in its own registers. The next step's K is loaded behind the scores' products, its V behind those of O.
//   * Rotation. cos and sin of a lane's pairs stay in registers and are turned on by 16 positions, found anew (to 1e-7) every 16 steps and where
//     positions jump.
//   * Work. A workgroup is one split of an item (16 rows of a request, a KV head), its four waves equal runs of the split's steps, merged
//     in LDS. There are as many splits as give the chip four workgroups a compute unit, of 32 steps or more each; one split writes
//     its rows, several leave partials for the merge.
//     Measured: 2.5e7 pairs (query row, slot) of D 128 in 61 us and 4e7 in 86, where the general kernel took 1477 and 966; the smallest call, 5 nodes x 8
//     heads behind 288 slots, 13.5 and 22.0 (half of it the launch and the first loads).
//   * A row that came out Inf or NaN is computed again by tree_row, which multiplies no slot that the row does not see.
#include "lanes.h"
#include "tree_common.h"

namespace mepic {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kRows = 16, kSlots = 16, kReseed = 16;

template <int D>
struct TreeF32Lds {
  float o[kWaves][kRows][D];
  float ml[kWaves][kRows][2];
  uint32_t path[MEPIC_TREE_MAX_NODES][kTreeWords];
  int16_t parent[MEPIC_TREE_MAX_NODES];
  int bad[kRows];
  TreeRowLds<kThreads> row;
};

template <int D>
__global__ __launch_bounds__(kThreads, 2) void tree_f32_kernel(const TreeF32Args m) {
  constexpr int kGranules = D / 16, kPairs = D / 8, kDims = D / 16;  // of a lane: granules and rotary pairs of a slot, tiles of dims
  __shared__ TreeF32Lds<D> lds;
  const AttnArgs& a = m.t.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), n16 = lane & 15, g = lane >> 4;
  const int P = a.P, logP = P == 16 ? 4 : 5, G = a.G;
  const int hk = blockIdx.x % a.Hkv, at = blockIdx.x / a.Hkv, split = at % m.splits, rt = at / m.splits % m.row_tiles, b = at / m.splits / m.row_tiles;
  TreeRequest r = tree_request(a, b);
  r.q0 = uni(r.q0); r.T = uni(r.T); r.kv_len = uni(r.kv_len); r.ctx = uni(r.ctx);
  const int nodes = min(r.T, m.t.max_q), rows_here = min(nodes * G - rt * kRows, kRows);
  if (rows_here <= 0) return;
  const int steps = (r.kv_len + kSlots - 1) / kSlots, per = (steps + kWaves * m.splits - 1) / (kWaves * m.splits);
  const int t0 = min(steps, (kWaves * split + wave) * per), t1 = min(steps, t0 + per);
  const size_t bt_row = (size_t)b * a.max_blocks;

  if ((long)kWaves * (split + 1) * per * kSlots > r.ctx) {  // the split has nodes among its slots
    if (tid < nodes) lds.parent[tid] = (int16_t)tree_parent(m.t.parents, r.q0, tid);
    __syncthreads();
    if (tid < nodes) {
      for (int w = 0; w < kTreeWords; ++w) lds.path[tid][w] = 0;
      for (int j = tid; j >= 0; j = lds.parent[j]) lds.path[tid][j >> 5] |= 1u << (j & 31);  // (numbers fall along a path)
    }
  }
  if (tid < kRows) lds.bad[tid] = 0;
  __syncthreads();

  const bool inter = a.interleaved;
  auto pair_index = [&](int p) { return inter ? 2 * (4 * (p / 2) + g) + p % 2 : 4 * (4 * (p / 4) + g) + p % 4; };
  auto cos_sin = [&](int pos, int p, float& c, float& s) { sincospif(2.f * turns_frac((float)pos, a.freq_hi[pair_index(p)], a.freq_lo[pair_index(p)]), &s, &c); };
  auto turn = [&](float4 (&x)[kGranules], const float (&c)[kPairs], const float (&s)[kPairs]) {
    auto one = [](float& lo, float& hi, float c, float s) {
      const float y = lo * c - hi * s;
      hi = hi * c + lo * s;
      lo = y;
    };
    if (inter) {
#pragma unroll
      for (int i = 0; i < kGranules; ++i) {
        one(x[i].x, x[i].y, c[2 * i], s[2 * i]);
        one(x[i].z, x[i].w, c[2 * i + 1], s[2 * i + 1]);
      }
    } else {
      constexpr int kHalf = kGranules / 2;
#pragma unroll
      for (int i = 0; i < kHalf; ++i) {
        one(x[i].x, x[i + kHalf].x, c[4 * i], s[4 * i]);
        one(x[i].y, x[i + kHalf].y, c[4 * i + 1], s[4 * i + 1]);
        one(x[i].z, x[i + kHalf].z, c[4 * i + 2], s[4 * i + 2]);
        one(x[i].w, x[i + kHalf].w, c[4 * i + 3], s[4 * i + 3]);
      }
    }
  };

  const int row = rt * kRows + n16, row_node = min(row / G, nodes - 1), head = row - row / G * G;
  float cs[kPairs], sn[kPairs];
  float4 q[kGranules];
  {
    const float* src = static_cast<const float*>(a.q) + ((size_t)(r.q0 + row_node) * a.Hq + (size_t)hk * G + head) * D;
#pragma unroll
    for (int i = 0; i < kGranules; ++i) __builtin_memcpy(&q[i], src + 4 * (4 * i + g), 16);
    const int pos = a.q_positions[r.q0 + row_node];
#pragma unroll
    for (int p = 0; p < kPairs; ++p) cos_sin(pos, p, cs[p], sn[p]);
    turn(q, cs, sn);
#pragma unroll
    for (int i = 0; i < kGranules; ++i) {
      q[i].x *= a.qk_scale_log2; q[i].y *= a.qk_scale_log2; q[i].z *= a.qk_scale_log2; q[i].w *= a.qk_scale_log2;
    }
  }

  floatx4 o[kDims];
#pragma unroll
  for (int dt = 0; dt < kDims; ++dt) o[dt] = floatx4{0.f, 0.f, 0.f, 0.f};
  float top = -INFINITY, sum = 0.f;
  if (t0 < t1) {
    float turn_c[kPairs], turn_s[kPairs];
#pragma unroll
    for (int p = 0; p < kPairs; ++p) cos_sin(kSlots, p, turn_c[p], turn_s[p]);
    const size_t page_bytes = (size_t)a.Hkv * D * P * 4, head_bytes = (size_t)hk * D * P * 4;
    const unsigned char* kp = static_cast<const unsigned char*>(a.k_pages) + head_bytes;
    const unsigned char* vp = static_cast<const unsigned char*>(a.v_pages) + head_bytes;
    float4 k[kGranules], v[kDims];
    auto block = [&](int t) { return bt_row + ((t * kSlots) >> logP); };
    auto load_k = [&](int t, int page) {
      const unsigned char* p = kp + (size_t)max(min(page, a.num_pages - 1), 0) * page_bytes + (size_t)(g * P + ((t * kSlots) & (P - 1)) + n16) * 16;
#pragma unroll
      for (int i = 0; i < kGranules; ++i) k[i] = *reinterpret_cast<const float4*>(p + (size_t)(4 * i * P) * 16);
    };
    auto load_v = [&](int t, int page) {
      const unsigned char* p = vp + (size_t)max(min(page, a.num_pages - 1), 0) * page_bytes + (size_t)(n16 * P + ((t * kSlots) & (P - 1)) + 4 * g) * 4;
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt) v[dt] = *reinterpret_cast<const float4*>(p + (size_t)(16 * dt * P) * 4);
    };
    int page = sload(a.block_tables, block(t0)), pos_now = 0;
    load_k(t0, page);
    load_v(t0, page);
#pragma unroll 1
    for (int t = t0; t < t1; ++t) {
      const int first = t * kSlots, n = first + n16, t2 = min(t + 1, t1 - 1);
      page = sload(a.block_tables, block(t2));
      int pos = n;
      if (a.block_positions) pos = sload(a.block_positions, block(t)) + (n & (P - 1));
      if (first + kSlots > r.ctx) {
        if (n >= r.ctx) pos = a.q_positions[r.q0 + max(min(n - r.ctx, r.T - 1), 0)];
        if (n >= r.kv_len) pos = pos_now + kSlots;
      }
      if (((t - t0) & (kReseed - 1)) != 0 && __all(pos == pos_now + kSlots)) {
#pragma unroll
        for (int p = 0; p < kPairs; ++p) {
          const float y = cs[p] * turn_c[p] - sn[p] * turn_s[p];
          sn[p] = sn[p] * turn_c[p] + cs[p] * turn_s[p];
          cs[p] = y;
        }
      } else {
#pragma unroll
        for (int p = 0; p < kPairs; ++p) cos_sin(pos, p, cs[p], sn[p]);
      }
      pos_now = pos;
      turn(k, cs, sn);
      floatx4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kGranules; ++i) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i].x, q[i].x, s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i].y, q[i].y, s1, 0, 0, 0);
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i].z, q[i].z, s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[i].w, q[i].w, s1, 0, 0, 0);
      }
      load_k(t2, page);
      float y[kSlots / 4];  // scores of slots first + 4 g + j and the lane's row
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] = s0[j] + s1[j];
      uint32_t word = low_bits(r.kv_len - first);  // slots that take part
      if (a.block_valid_mask) word &= (uint32_t)sload(reinterpret_cast<const int32_t*>(a.block_valid_mask), block(t)) >> (first & (P - 1));
      word &= 0xffffu;
      if (word != 0xffffu || first + kSlots > r.ctx) {
        const uint32_t bits = (word & path_bits(lds.path[row_node], first, r.ctx)) >> (4 * g);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (bits >> j) & 1u ? y[j] : -INFINITY;
        const uint32_t keep = word >> (4 * g);  // slots that take no part may hold anything
#pragma unroll
        for (int dt = 0; dt < kDims; ++dt) {
          v[dt].x = keep & 1u ? v[dt].x : 0.f;
          v[dt].y = keep & 2u ? v[dt].y : 0.f;
          v[dt].z = keep & 4u ? v[dt].z : 0.f;
          v[dt].w = keep & 8u ? v[dt].w : 0.f;
        }
      }
      const float most = fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3]));
      if (__any(most > top + 8.f)) {  // (the reference maximum lags by up to 8: weights stay below 2^8)
        const float now = fmaxf(top, max_over_kgroups(most));
        const float f = now == top ? 1.f : __builtin_amdgcn_exp2f(top - now);
        top = now;
        sum *= f;
#pragma unroll
        for (int dt = 0; dt < kDims; ++dt)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[dt][i] *= f;
      }
      const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] = __builtin_amdgcn_exp2f(y[j] - ref);
        sum += y[j];
      }
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt) {
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[dt].x, y[0], o[dt], 0, 0, 0);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[dt].y, y[1], o[dt], 0, 0, 0);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[dt].z, y[2], o[dt], 0, 0, 0);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[dt].w, y[3], o[dt], 0, 0, 0);
      }
      load_v(t2, page);
    }
  }

  // ---- the waves' runs merged ----
  sum = sum_over_kgroups(sum);
  if (g == 0) {
    lds.ml[wave][n16][0] = top;
    lds.ml[wave][n16][1] = sum;
  }
#pragma unroll
  for (int dt = 0; dt < kDims; ++dt) *reinterpret_cast<floatx4*>(&lds.o[wave][n16][16 * dt + 4 * (g ^ (n16 & 3))]) = o[dt];
  __syncthreads();
  const size_t part = ((size_t)((b * m.row_tiles + rt) * (size_t)m.splits + split) * a.Hkv + hk) * kRows;
  for (int u = tid; u < rows_here * (D / 4); u += kThreads) {
    const int in = u / (D / 4), quad = u % (D / 4);
    float mx = -INFINITY, den = 0.f;
    floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) mx = fmaxf(mx, lds.ml[w][in][0]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mi = lds.ml[w][in][0], li = lds.ml[w][in][1];
      if (mi == -INFINITY && li == 0.f) continue;  // no slot took part
      const float f = mi == mx ? 1.f : __builtin_amdgcn_exp2f(mi - mx);
      const floatx4 y = *reinterpret_cast<const floatx4*>(&lds.o[w][in][4 * (quad ^ (in & 3))]);
      den += f * li;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] += f * y[j];
    }
    if (m.splits > 1) {
      *reinterpret_cast<floatx4*>(m.part_o + (part + in) * D + 4 * quad) = x;
      if (quad == 0) *reinterpret_cast<float2*>(m.part_ml + (part + in) * 2) = make_float2(mx, den);
    } else {
      const int all = rt * kRows + in, node = all / G;
      const float inv = den != 0.f ? 1.f / den : 0.f;
      const floatx4 w = x * inv;
      __builtin_memcpy(static_cast<float*>(a.out) + ((size_t)(r.q0 + node) * a.Hq + (size_t)hk * G + all - node * G) * D + 4 * quad, &w, 16);
      if (!((x[0] + x[1] + x[2] + x[3]) * 0.f + den * 0.f == 0.f)) lds.bad[in] = 1;
    }
  }
  __syncthreads();
  if (m.splits > 1) return;
  for (int in = 0; in < rows_here; ++in) {
    if (!lds.bad[in]) continue;
    const int all = rt * kRows + in, node = all / G;
    tree_row<MEPIC_F32, kThreads>(m.t, lds.row, r, b, node, hk * G + all - node * G);
  }
}

// Rows of calls with several splits: a wave has one row, a lane two dims (D 64: one).
template <int D>
__global__ __launch_bounds__(kThreads) void tree_f32_merge_kernel(const TreeF32Args m) {
  constexpr int kPer = D / 64;
  __shared__ int bad[kWaves];
  __shared__ TreeRowLds<kThreads> lds;
  const AttnArgs& a = m.t.a;
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), row = blockIdx.x * kWaves + wave;
  const int t = row / a.Hq, hq = row - t * a.Hq, hk = hq / a.G;
  const int b = row < a.n_q * a.Hq ? request_of(a.cu_q_lens, a.B, t) : -1;
  const int node = b < 0 ? 0 : t - tree_request(a, b).q0;
  const bool here = b >= 0 && node < m.t.max_q;
  if (lane == 0) bad[wave] = 0;
  if (here) {
    const int all = node * a.G + hq - hk * a.G;
    const size_t first = (size_t)(b * m.row_tiles + all / kRows) * m.splits;
    auto part = [&](int s) { return ((first + s) * a.Hkv + hk) * kRows + all % kRows; };
    float mx = -INFINITY, den = 0.f, x[kPer] = {};
    for (int s = 0; s < m.splits; ++s) mx = fmaxf(mx, m.part_ml[2 * part(s)]);
#pragma unroll 4
    for (int s = 0; s < m.splits; ++s) {
      const size_t p = part(s);
      const float mi = m.part_ml[2 * p], li = m.part_ml[2 * p + 1];
      const float f = mi == -INFINITY && li == 0.f ? 0.f : mi == mx ? 1.f : __builtin_amdgcn_exp2f(mi - mx);
      den += f * li;
#pragma unroll
      for (int i = 0; i < kPer; ++i) x[i] += f * m.part_o[p * D + kPer * lane + i];
    }
    const float inv = den != 0.f ? 1.f / den : 0.f;
    float odd = den * 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      static_cast<float*>(a.out)[(size_t)row * D + kPer * lane + i] = x[i] * inv;
      odd += x[i] * 0.f;
    }
    if (!(odd == 0.f)) bad[wave] = 1;
  }
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) {
    if (!bad[w]) continue;
    const int r = blockIdx.x * kWaves + w, tok = r / a.Hq, req = request_of(a.cu_q_lens, a.B, tok);
    const TreeRequest rq = tree_request(a, req);
    tree_row<MEPIC_F32, kThreads>(m.t, lds, rq, req, tok - rq.q0, r - tok * a.Hq);
  }
}

template <int D>
void launch(const TreeF32Args& m, unsigned workgroups, hipStream_t s) {
  tree_f32_kernel<D><<<workgroups, kThreads, 0, s>>>(m);
  if (m.splits > 1) tree_f32_merge_kernel<D><<<((unsigned)m.t.a.n_q * m.t.a.Hq + kWaves - 1) / kWaves, kThreads, 0, s>>>(m);
}

}  // namespace

TreePlan tree_f32_plan(const TreeArgs& t, int max_kv) {
  const AttnArgs& a = t.a;
  TreePlan p{};
  if (a.max_blocks == 0 || a.num_pages == 0 || a.B == 0) return p;  // (no page to read)
  const long row_tiles = ((long)t.max_q * a.G + kRows - 1) / kRows, items = (long)a.B * row_tiles * a.Hkv;
  if (items > INT_MAX / 2) return p;
  const long steps = (max_kv + kSlots - 1) / kSlots, wanted = (4L * device_compute_units() + items - 1) / items, most = (steps + 31) / 32;
  p.rows = kRows;
  p.row_tiles = (int)row_tiles;
  p.splits = (int)(wanted < most ? wanted : most > 1 ? most : 1);
  if (p.splits > 1) p.bytes = (size_t)items * p.splits * kRows * (a.D + 2) * sizeof(float);
  return p;
}

hipError_t launch_tree_f32(const TreeArgs& t, const TreePlan& pl, void* workspace, hipStream_t s) {
  const AttnArgs& a = t.a;
  TreeF32Args m{};
  m.t = t;
  m.row_tiles = pl.row_tiles;
  m.splits = pl.splits;
  const size_t items = (size_t)a.B * pl.row_tiles * a.Hkv;
  m.part_o = static_cast<float*>(workspace);
  m.part_ml = m.part_o + items * pl.splits * kRows * a.D;
  const unsigned workgroups = (unsigned)(items * pl.splits);
  if (a.D == 128) launch<128>(m, workgroups, s);
  else launch<64>(m, workgroups, s);
  return hipGetLastError();
}

}  // namespace mepic
