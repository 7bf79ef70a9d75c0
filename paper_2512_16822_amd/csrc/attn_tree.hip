// Attention of a tree of drafted tokens: the general kernel (every case the call allows, in plain fp32 arithmetic, one workgroup per
// output row: 64 requests x 4.3 K bf16 slots x 64 rows take 10.6 ms, bound by sines and cosines of each row's own), and of the
// matrix-core kernels for bf16 and e4m3 pages the plan, the merge of rows that several workgroups share, and the dispatch.
#include "merge_partials.h"
#include "tree_common.h"

namespace mepic {
namespace {

constexpr int kRowThreads = 256;

template <int KV>
__global__ __launch_bounds__(kRowThreads) void tree_general_kernel(const TreeArgs ta) {
  __shared__ TreeRowLds<kRowThreads> lds;
  const int t = blockIdx.x / ta.a.Hq, hq = blockIdx.x % ta.a.Hq;
  const int b = request_of(ta.a.cu_q_lens, ta.a.B, t);
  if (b < 0) return;
  const TreeRequest r = tree_request(ta.a, b);
  if (t - r.q0 >= ta.max_q) return;
  tree_row<KV, kRowThreads>(ta, lds, r, b, t - r.q0, hq);
}

// Rows whose item was cut: the partials of workgroups first .. last, the first one's in its second slot, the others' in their first. Groups of
// D / 4 threads, a thread four dims; each group has a row of its own, or (kOneRow) all take every kGroups-th partial of one row. Few rows have many
// partials each and leave most of the chip idle, many rows are bound by launching their workgroups: us of both kernels, with a workgroup per row and per eight, 8
// nodes x 32 heads of one request 19.3 and 22.2, of four 31.4 and 31.4; 16 x 32 of 8 requests 52.2 and 47.5, of 32 117 and 94.
template <int KV, int D, bool kOneRow>
__global__ __launch_bounds__(kRowThreads) void tree_merge_kernel(const TreeMfmaArgs m, int rows) {
  constexpr int kCols = D / 4, kGroups = kRowThreads / kCols;
  __shared__ float4 num_s[kGroups][kCols];
  __shared__ float2 ml_s[kGroups];
  __shared__ int bad[kGroups];
  __shared__ TreeRowLds<kRowThreads> lds;
  const AttnArgs& a = m.t.a;
  const int grp = threadIdx.x / kCols, col = threadIdx.x % kCols;
  const int row = kOneRow ? blockIdx.x : blockIdx.x * kGroups + grp;
  const int t = row / a.Hq, hq = row - t * a.Hq, hk = hq / a.G;
  const bool here = row < a.n_q * a.Hq && t < a.cu_q_lens[a.B];
  int4 w = make_int4(0, 0, 0, 0);
  if (here) w = m.row_wgs[(size_t)t * a.G + hq - hk * a.G];
  // (a request that breaks max_q_len has rows nobody wrote: whatever is there forms no address outside the workspace)
  const int first = min(max(w.x, 0), m.groups - 1), last = min(max(w.y, first), m.groups - 1), in = min(max(w.z, 0), rows - 1);
  const bool cut = here && last > first;
  if (kOneRow && !cut) return;
  float top = -INFINITY, den = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  auto add = [&](const float2& e, const float4& y) {
    if (e.x == -INFINITY && e.y == 0.f) return;  // no slot took part
    const float now = fmaxf(top, e.x);
    const float f = now == top ? 1.f : __builtin_amdgcn_exp2f(top - now), u = now == e.x ? 1.f : __builtin_amdgcn_exp2f(e.x - now);
    top = now;
    den = den * f + u * e.y;
    x.x = x.x * f + u * y.x; x.y = x.y * f + u * y.y; x.z = x.z * f + u * y.z; x.w = x.w * f + u * y.w;
  };
  auto part = [&](int s) { return (((size_t)s * a.Hkv + hk) * 2 + (s == first ? 1 : 0)) * rows + in; };
  if (cut) {
    constexpr int kStep = kOneRow ? kGroups : 1;
    for (int s = first + (kOneRow ? grp : 0); s <= last; s += 4 * kStep) {
      float2 e[4];
      float4 y[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const size_t p = part(min(s + i * kStep, last));
        e[i] = *reinterpret_cast<const float2*>(m.part_ml + 2 * p);
        y[i] = *reinterpret_cast<const float4*>(m.part_o + p * D + 4 * col);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (s + i * kStep <= last) add(e[i], y[i]);
    }
  }
  if constexpr (kOneRow) {
    num_s[grp][col] = x;
    if (col == 0) ml_s[grp] = make_float2(top, den);
    __syncthreads();
    top = -INFINITY; den = 0.f;
    x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < kGroups; ++i) add(ml_s[i], num_s[i][col]);
  }
  if (col == 0) bad[grp] = 0;
  __syncthreads();
  if (cut && (!kOneRow || grp == 0)) {
    const float inv = den != 0.f ? 1.f / den : 0.f;
    uint2 v;
    v.x = pack2_bf16(x.x * inv, x.y * inv);
    v.y = pack2_bf16(x.z * inv, x.w * inv);
    __builtin_memcpy(static_cast<uint16_t*>(a.out) + (size_t)row * D + 4 * col, &v, 8);
    const float odd = (x.x + x.y + x.z + x.w) * 0.f + den * 0.f;
    if (!(odd == 0.f)) bad[grp] = 1;
  }
  __syncthreads();
  for (int i = 0; i < (kOneRow ? 1 : kGroups); ++i) {
    if (!bad[i]) continue;
    const int r = kOneRow ? (int)blockIdx.x : (int)blockIdx.x * kGroups + i, tok = r / a.Hq, b = request_of(a.cu_q_lens, a.B, tok);
    if (b < 0) continue;
    const TreeRequest rq = tree_request(a, b);
    if (tok - rq.q0 < m.t.max_q) tree_row<KV, kRowThreads>(m.t, lds, rq, b, tok - rq.q0, r - tok * a.Hq);
  }
}

template <int KV, int D>
void launch_merge(const TreeMfmaArgs& m, int rows, hipStream_t s) {
  const int n = m.t.a.n_q * m.t.a.Hq;
  if (n <= 1024) {
    tree_merge_kernel<KV, D, true><<<n, kRowThreads, 0, s>>>(m, rows);
  } else {
    constexpr int per = kRowThreads / (D / 4);
    tree_merge_kernel<KV, D, false><<<(n + per - 1) / per, kRowThreads, 0, s>>>(m, rows);
  }
}

}  // namespace

TreePlan tree_mfma_plan(const TreeArgs& t, int max_kv) {
  const AttnArgs& a = t.a;
  TreePlan p{};
  if (a.max_blocks == 0 || a.num_pages == 0 || a.B == 0) return p;  // (no page to read)
  // Rows of a tile: a tile's keys are staged once for all of them, so the fewest tiles that hold a request's rows, unless most of the
  // requests fill far less than the largest one does. us a call with tiles of 32, 64, 128 and 256 rows: 32 requests x 4.3 K bf16 slots, 32 rows each
  // 82, 90, -, 137; 64 rows 152, 106, -, 146; 4 - 80 rows 149, 119, -, 142; 68 - 128 rows each 177 - 192 with 64 and 193 - 210 with 128 (two tiles in windows
  // beat one without); 4 - 160 rows -, 177, -, 184; 4 - 192 -, 202, -, 190; 192 each -, 300, -, 225. e4m3 has less to stage and its scores' scales to
  // apply: 68 - 128 rows each 192 - 205 with 64 and 157 - 173 with 128; 4 - 160 rows -, 184, 183, 192; 128 requests of 2 - 33 K slots, 21 - 84 rows, -, 821, 932.
  const long most = (long)t.max_q * a.G, mean = (long)a.n_q * a.G / a.B;  // rows of a request, at most and on average
  if (most <= 32) p.rows = 32;
  else if (most <= 64 || mean <= 64) p.rows = 64;
  else if (a.kv_dtype == MEPIC_F8E4M3) p.rows = most <= 128 || mean <= 128 ? 128 : 256;
  else p.rows = most <= 128 || mean <= 96 ? 64 : 256;
  const int cus = device_compute_units();
  // (32 rows leave little to do per slot: one workgroup of eight waves stages twice the tile per barrier, 8 x 65 K slots 376 us, two of four waves 390)
  const int resident = p.rows == 32 || p.rows == 256 ? cus : 2 * cus;  // workgroups of eight and of four waves
  p.groups = resident / a.Hkv > 1 ? resident / a.Hkv : 1;
  const long tiles = (max_kv + 63) / 64;
  // (the work is counted in 32 bits, whatever lengths the device brings: the table's width bounds them, max_kv_len is the caller's word)
  const long widest = ((long)a.max_blocks * a.P + 63) / 64;
  if (((long)a.n_q * a.G / p.rows + a.B + 1) * (widest + 8) > (1L << 30)) return TreePlan{};
  // Short contexts are not cut, there is nothing to merge then: us uncut and cut, 4 requests of 80 slots 12.5 and 23.0, of 470 17.5 and 18.7, of 920 24.5 and
  // 20.0; 32 of 470 21.7 and 27.1. A run has 256 slots or more: runs of 128, 256 and 512 take 17.0, 18.6, 20.6 us for one request of 1.2 K, 22.2,
  // 21.6, 28.4 for four of 1.7 K, 33.9, 33.2, 33.6 for four of 4.3 K.
  p.whole = tiles <= 8;
  p.min_slots = 256;
  if (!p.whole)
    p.bytes = (size_t)p.groups * a.Hkv * 2 * p.rows * (a.D + 2) * sizeof(float) + (size_t)a.n_q * a.G * sizeof(int4);
  return p;
}

hipError_t launch_tree_mfma(const TreeArgs& t, const TreePlan& pl, void* workspace, hipStream_t s) {
  const AttnArgs& a = t.a;
  TreeMfmaArgs m{};
  m.t = t;
  m.groups = pl.groups; m.min_slots = pl.min_slots; m.whole = pl.whole;
  const size_t parts = (size_t)pl.groups * a.Hkv * 2 * pl.rows;
  m.row_wgs = static_cast<int4*>(workspace);
  m.part_o = reinterpret_cast<float*>(m.row_wgs + (size_t)a.n_q * a.G);
  m.part_ml = m.part_o + parts * a.D;
  const bool fp8 = a.kv_dtype == MEPIC_F8E4M3;
  hipError_t e = fp8 ? launch_tree_tiles_fp8(pl.rows, m, s) : launch_tree_tiles_bf16(pl.rows, m, s);
  if (a.timing_stop) (void)hipEventRecord(reinterpret_cast<hipEvent_t>(a.timing_stop), s);
  if (e != hipSuccess || pl.whole) return e;
  if (fp8 && a.D == 128) launch_merge<MEPIC_F8E4M3, 128>(m, pl.rows, s);
  else if (fp8) launch_merge<MEPIC_F8E4M3, 64>(m, pl.rows, s);
  else if (a.D == 128) launch_merge<MEPIC_BF16, 128>(m, pl.rows, s);
  else launch_merge<MEPIC_BF16, 64>(m, pl.rows, s);
  return hipGetLastError();
}

hipError_t launch_tree_general(const TreeArgs& t, hipStream_t s) {
  const dim3 grid((unsigned)t.a.n_q * t.a.Hq);
  if (t.a.kv_dtype == MEPIC_F32) tree_general_kernel<MEPIC_F32><<<grid, kRowThreads, 0, s>>>(t);
  else if (t.a.kv_dtype == MEPIC_BF16) tree_general_kernel<MEPIC_BF16><<<grid, kRowThreads, 0, s>>>(t);
  else tree_general_kernel<MEPIC_F8E4M3><<<grid, kRowThreads, 0, s>>>(t);
  return hipGetLastError();
}

}  // namespace mepic
