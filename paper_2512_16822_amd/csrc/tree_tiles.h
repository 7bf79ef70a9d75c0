// Attention of a tree of drafted tokens on the matrix cores, bf16 and e4m3 pages: the kernel, a template that the attn_tree_*.hip
// files instantiate.
//
// A verification step brings R = nodes x (Hq / Hkv) query rows per KV head to the same context: 8 to 512 where decode has 1 to 16. So
// a key is rotated once per tile of rows and shared through LDS. What bounds it is vector work: of 64 requests x 4.3 K slots x 64 rows (163 us, 443
// TFLOP/s) the vector units are busy 55 % of the time, with two waves a SIMD that wait 29 % of theirs, mostly at a tile's barrier, LDS 37 %,
// the matrix cores 22 %. With 24 rows, 8 x 65 K slots, it is memory: 376 us, 5.7 TB/s.
//   * Work. An item is a tile of kRows rows of one request; its keys come in tiles of kTile = 16 kWaves slots. The (item, tile) pairs of a KV head
//     form one sequence that the head's workgroups cut into equal runs (an item's start counts for some tiles too); a row cut in two or more goes through partials and
//     tree_merge_kernel, any other is written directly. With four waves two workgroups share a compute unit and fill each other's waits (64 rows,
//     when it was chosen: 178 us; one of eight waves and twice the tile 191).
//   * Staging. A wave has an octet of rotary pairs (or two), a lane one slot or two. K goes to LDS as fp16 in operand order, V as matrix operands too (e4m3
//     widened to fp16, which holds the codes exactly); the loads of the next tile are in flight during the products of this one, ids,
//     masks and scales ahead of keys and values.
//   * Rotation, in general: cos and sin of its slot's position stay in a lane's registers in fp32 and are turned on from slot to slot (the turn is
//     the same for a wave: scalar registers), found anew every 16 tiles and where positions jump. Tiles of 64 rows without masks, positions
//     or interleaving (kWindows): a window of two tiles starts at position 0 for its keys, whose cos and sin are then the same in every window and kept as packed fp16,
//     and the queries, kept in fp32, are turned back by a window's length instead: 171 us against 182 when both were
//     measured, at 2 us more before a workgroup's first tile. With 32 rows there is too little else to do for that to pay: 8 x 65 K slots 376 us without, 407 with.
//   * Products. S^T[32 slots x 16 rows] = K Q^T with v_mfma_f32_16x16x32_f16 and O^T[dims x rows] += V^T P^T: a lane owns one row, so
//     sums, maxima and rescaling are its own. Slots are laid out so that the scores a lane gets are the eight consecutive slots its
//     operand of P^T needs. kGroups groups of waves take 16 kTiles rows each; where several waves share a group's rows, they have different slots
//     and are merged in LDS at the end of a run.
//   * Precision. Query rows are scaled by a power of two to at most 1 and keys times 16 (kWindows and e4m3 codes: as they are), both in fp16: 11
//     significant bits where bf16 has 8; a key beyond 2896 (46340) gives an infinite score, which marks the row. P is bf16 next to bf16 V, fp16
//     next to e4m3 V, where the exponent of the page's V scale joins the score and its mantissa P. Sums and O are fp32. The reference maximum
//     of a row lags by up to 8 (log2 units).
//   * A marked row, or one that came out Inf or NaN, is computed again by tree_row.
#pragma once
#include <cstddef>
#include <type_traits>

#include "lanes.h"
#include "tree_common.h"

namespace mepic {

constexpr int kReseed = 16;  // tiles after which cos and sin are found anew

template <int kWaves>
struct TreeLdsTail {  // behind the two tile buffers
  TreeArgs args;  // what the loop over tiles does not need is read from here: kernel arguments would fill the scalar registers
  float *part_o, *part_ml;
  uint32_t path[MEPIC_TREE_MAX_NODES][kTreeWords];
  int16_t parent[MEPIC_TREE_MAX_NODES];
  int node_pos[MEPIC_TREE_MAX_NODES];
  float2 back[kMaxHalfD];  // cos and sin of a window's turn
  float ml[kWaves][32][2];  // maxima and sums, where several waves share a row's slots
  uint32_t bad[kWaves];  // a bit a row: to be computed again
  int scan[kWaves * 2];
  int found[2];
  TreeRowLds<kWaves * 64> row;
};

// Two tiles of K and V operands and the tail: with four waves two workgroups of D 128 fit a compute unit.
template <int D, int kWaves> constexpr size_t tree_lds_bytes() { return 2 * (size_t)(16 * kWaves) * D * 2 * 2 + sizeof(TreeLdsTail<kWaves>); }
static_assert(2 * tree_lds_bytes<128, 4>() <= 160 * 1024);

__device__ __forceinline__ uint32_t pack2_f16(float lo, float hi) {
  const f32x2 v = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// Two e4m3 codes of a word (the low or the high two) as packed fp16, exactly.
__device__ __forceinline__ uint32_t f16_of_e4m3(uint32_t w, bool high) {
  return __builtin_bit_cast(uint32_t, high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
}

template <bool kFp8, int D, int kWaves, int kGroups, int kTiles, bool kPlain>
__global__ __launch_bounds__(kWaves * 64, 2) void tree_tiles_kernel(const TreeMfmaArgs m) {
  constexpr int kThreads = kWaves * 64, kTile = 16 * kWaves;  // slots of a tile
  constexpr int kRows = kGroups * kTiles * 16, kSlotGroups = kWaves / kGroups, kSubs = kTile / 32 / kSlotGroups;
  static_assert(kSubs >= 1, "a wave has at least 32 slots of a tile");
  constexpr int kSteps = D / 32, kDims = D / 16;          // products per score, 16-dim tiles of O
  constexpr int E = kFp8 ? 1 : 2, X = 16 / E, DX = D / X;  // bytes per element, elements per granule
  // a thread stages kHalves octets of dims: of D 128 eight waves have one octet of two slots each, four waves two octets of one slot
  constexpr int kHalves = D / 64, kSlotStep = kWaves == 8 && D == 128 ? 64 : 0, kOctetStep = kWaves == 4 && D == 128 ? 4 : 0;
  constexpr int kTurn = kSlotStep ? kSlotStep : kTile;  // positions from a thread's slot to its next
  constexpr int kSets = kOctetStep ? kHalves : 1;       // octets whose cos and sin a thread has
  constexpr int kKeyBytes = kTile * D * 2, kTileBytes = 2 * kKeyBytes;
  constexpr int kVGranules = 16 * D * E / 16 / 64;        // 16-byte pieces of V per lane and tile
  constexpr int kRing = kTiles == 1 && D == 128 ? 8 : 4;  // operands in flight: some 150 clocks a read, 16 a product
  constexpr bool kWindows = kPlain && kTiles == 1 && kSlotGroups == 1;  // keys turned from the start of a window of two tiles (see Staging)
  // What the start of an item (queries, paths, first loads) counts for in tiles, where workgroups are given equal parts: 256 slots' worth, which a tile of
  // 256 rows takes as long for as for a start. Without it whoever has the joint of two requests ends last: 4 x 1.7 K slots 26.2 us and 20.9, 16 x 0.5 - 3.1 K in
  // a whole step 73.0 and 68.5, 128 x 2 - 33 K e4m3 825 and 810; 256 rows 332 without, 336 with.
  constexpr int kStart = kRows == 256 ? 0 : 256 / kTile;
  constexpr float kKeyFactor = kFp8 || kWindows ? 1.f : 16.f;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];
  TreeLdsTail<kWaves>& tail = *reinterpret_cast<TreeLdsTail<kWaves>*>(lds + 2 * kTileBytes);
  const TreeArgs& ta = tail.args;
  const AttnArgs& a = ta.a;
  const AttnArgs& hot = m.t.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), n16 = lane & 15, g = lane >> 4;
  const int hk = blockIdx.x % hot.Hkv, wg = blockIdx.x / hot.Hkv, G = hot.G, P = hot.P, logP = P == 16 ? 4 : 5;
  const int rg = wave % kGroups, sg = wave / kGroups;

  if (tid == 0) {
    __builtin_memcpy(&tail.args.a, &m.t.a, offsetof(AttnArgs, freq_hi));
    tail.args.parents = m.t.parents;
    tail.args.max_q = m.t.max_q;
    tail.part_o = m.part_o;
    tail.part_ml = m.part_ml;
  }
  if (tid < kWaves) tail.bad[tid] = 0;
  if (tid < D / 2) {
    tail.args.a.freq_hi[tid] = m.t.a.freq_hi[tid];
    tail.args.a.freq_lo[tid] = m.t.a.freq_lo[tid];
    if (kWindows) {
      const float f = turns_frac(2.f * kTile, m.t.a.freq_hi[tid], m.t.a.freq_lo[tid]);
      tail.back[tid] = make_float2(__builtin_amdgcn_cosf(f), __builtin_amdgcn_sinf(f));
    }
  }
  __syncthreads();

  // ---- this workgroup's run: [begin, end) of the (item, tile) pairs of all requests ----
  auto cost_of = [&](int b, int& tiles, int& items) {
    const TreeRequest r = tree_request(a, b);
    tiles = max((r.kv_len + kTile - 1) / kTile, 1);
    items = (min(r.T, ta.max_q) * G + kRows - 1) / kRows;
    return m.whole ? items : items * (tiles + kStart);
  };
  // inclusive prefix sums of the costs of kThreads requests; returns their total
  auto scan_costs = [&](int b0, int& incl, int& cost) {
    int tiles, items;
    cost = b0 + tid < a.B ? cost_of(b0 + tid, tiles, items) : 0;
    incl = cost;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int y = __shfl_up(incl, o);
      if (lane >= o) incl += y;
    }
    if (lane == 63) tail.scan[wave] = incl;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const int x = tail.scan[w];
      if (w < wave) before += x;
      total += x;
    }
    incl += before;
    __syncthreads();
    return total;
  };
  int incl, cost, total = scan_costs(0, incl, cost);
  for (int b0 = kThreads; b0 < a.B; b0 += kThreads) {
    int i2, c2;
    total += scan_costs(b0, i2, c2);
  }
  const int per = max((total + m.groups - 1) / m.groups, m.whole ? 1 : m.min_slots / kTile);
  int at = wg * per;
  const int end = min(total, at + per);
  if (at >= end) return;
  int b = 0, before = 0;  // the request of `at`, and the cost of those in front of it
  {
    int base = 0, sum = a.B > kThreads ? scan_costs(0, incl, cost) : total;
    for (int b0 = 0;; ) {
      if (cost > 0 && base + incl - cost <= at && at < base + incl) {
        tail.found[0] = b0 + tid;
        tail.found[1] = base + incl - cost;
      }
      if (at < base + sum) break;
      base += sum;
      b0 += kThreads;
      sum = scan_costs(b0, incl, cost);
    }
    __syncthreads();
    b = uni(tail.found[0]);
    before = uni(tail.found[1]);
  }

  // ---- what a thread stages: the eight pairs of octet pc (the wave's) of slot sl, then those kOctetStep octets and kSlotStep slots on;
  // in LDS a slot lies at `place` ----
  const int pc = wave & (D / 16 - 1), place = (D == 64 && kWaves == 8 ? (wave >> 2) * 64 : 0) + lane;
  const int sl = (place & ~31) | ((place & 12) << 1) | ((place & 16) >> 2) | (place & 3);
  float turn_c[kSets][8], turn_s[kSets][8];  // the turn by kTurn positions
  const bool inter = !kPlain && hot.interleaved;
  auto freq_index = [&](int i, int e) {
    const int c = pc + i * kOctetStep;
    return !inter ? 8 * c + e : e < 4 ? 4 * c + e : D / 4 + 4 * c + e - 4;
  };
#pragma unroll
  for (int i = 0; i < kSets; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = turns_frac((float)kTurn, a.freq_hi[freq_index(i, e)], a.freq_lo[freq_index(i, e)]);
      turn_c[i][e] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(__builtin_amdgcn_cosf(f))));
      turn_s[i][e] = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(__builtin_amdgcn_sinf(f))));
    }
  // kWindows: cos and sin of a thread's slots of a window, for two pairs a register
  f16x2 win_c[kWindows ? 2 * kHalves : 1][4], win_s[kWindows ? 2 * kHalves : 1][4];
  bool win_kept = false;
  auto keep_window = [&]() {  // [tile of the window * kHalves + half]
#pragma unroll
    for (int i = 0; i < kSets; ++i) {
      float c[8], s[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = turns_frac((float)sl, a.freq_hi[freq_index(i, e)], a.freq_lo[freq_index(i, e)]);
        c[e] = __builtin_amdgcn_cosf(f);
        s[e] = __builtin_amdgcn_sinf(f);
      }
#pragma unroll
      for (int h = i; h < (kWindows ? 2 * kHalves : 1); h += kSets) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          win_c[h][j] = __builtin_bit_cast(f16x2, pack2_f16(c[2 * j], c[2 * j + 1]));
          win_s[h][j] = __builtin_bit_cast(f16x2, pack2_f16(s[2 * j], s[2 * j + 1]));
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float y = c[e] * turn_c[i][e] - s[e] * turn_s[i][e];
          s[e] = s[e] * turn_c[i][e] + c[e] * turn_s[i][e];
          c[e] = y;
        }
      }
    }
    win_kept = true;
  };
  const int v_page = wave >> (logP - 4), v_first = (wave & ((P >> 4) - 1)) * (64 * kVGranules);
  // a lane's pieces of V: X consecutive slots (part v_part of a page's) of one dim, one or two operands of eight. In LDS operand (octet of
  // slots, dim) lies at octet * D + (dim ^ twist): lanes that write together, of one dim and several octets, hit different banks
  const int v_per = P / X, v_part = (v_first + lane) & (v_per - 1), v_dim = (v_first + lane) >> (v_per == 1 ? 0 : v_per == 2 ? 1 : 2);
  const int v_stride = 64 / v_per * 16;  // (the dims of one lane are multiples of 16 apart: the twist is the same)
  // (a read of 16 bytes a lane serves lanes 0-3, 12-15, 20-23, 24-27 together, then 4-11, 16-19, 28-31, and so on: octets 2i and 2i + 1 must keep
  // dims 0-3 and 12-15 apart from 4-11, which 12 does; a write serves 16 consecutive lanes, two or four octets)
  auto twist_of = [&](int octet) { return (octet & 1 ? 12 : 0) ^ (octet & 2 ? 4 : 0); };
  int v_dst[X / 8];
#pragma unroll
  for (int h = 0; h < X / 8; ++h) {
    const int octet = ((v_page << logP) >> 3) + v_part * (X / 8) + h;
    v_dst[h] = kKeyBytes + (octet * D + (v_dim ^ twist_of(octet))) * 16;
  }
  const int k_src = (g * kTile + n16) * 16, v_src = kKeyBytes + (g * D + (n16 ^ twist_of(g))) * 16;  // a lane's first operands
  const size_t page_bytes = (size_t)hot.Hkv * D * P * E, head_bytes = (size_t)hk * D * P * E;
  const unsigned char* kp = static_cast<const unsigned char*>(hot.k_pages) + head_bytes;
  const unsigned char* vp = static_cast<const unsigned char*>(hot.v_pages) + head_bytes;

  while (at < end) {
    TreeRequest r = tree_request(a, b);
    r.q0 = uni(r.q0); r.T = uni(r.T); r.kv_len = uni(r.kv_len); r.ctx = uni(r.ctx);
    int tiles, items;
    const int mine = uni(cost_of(b, tiles, items));
    tiles = uni(tiles);
    if (at >= before + mine) {  // on to the next request
      before += mine;
      if (++b >= a.B) return;
      continue;
    }
    const int units = m.whole ? 1 : tiles + kStart, rt = (at - before) / units, unit = at - before - rt * units;
    const int stop = min(units, unit + end - at);  // the run's units of the item are unit .. stop - 1
    const int t0 = m.whole ? 0 : max(unit - kStart, 0), t1 = m.whole ? tiles : stop - kStart;
    at += stop - unit;
    if (t1 <= t0) continue;  // none of its tiles
    const int n_rows = min(r.T, ta.max_q) * G - rt * kRows;  // rows from the item's first to the request's last
    const size_t bt_row = (size_t)b * a.max_blocks;

    // rows that other workgroups share: which ones (head 0 says so for all)
    if (!m.whole && t0 == 0 && hk == 0) {
      const int last = (before + (rt + 1) * units - 1) / per;
      for (int i = tid; i < min(n_rows, kRows); i += kThreads) {
        m.row_wgs[(size_t)r.q0 * G + rt * kRows + i] = make_int4(wg, last, i, b);
      }
    }
    // paths, where the run has nodes among its slots
    const bool nodes_here = t1 * kTile > r.ctx;
    if (nodes_here) {
      const int T = min(r.T, MEPIC_TREE_MAX_NODES);
      if (tid < T) {
        tail.parent[tid] = (int16_t)tree_parent(ta.parents, r.q0, tid);
        tail.node_pos[tid] = a.q_positions[r.q0 + tid];
      }
      __syncthreads();
      if (tid < T) {
#pragma unroll
        for (int w = 0; w < kTreeWords; ++w) tail.path[tid][w] = 0;
        int word = tid >> 5;
        uint32_t bits = 0;
        for (int j = tid; j >= 0; j = tail.parent[j]) {  // (numbers fall along a path)
          if ((j >> 5) != word) {
            tail.path[tid][word] = bits;
            word = j >> 5;
            bits = 0;
          }
          bits |= 1u << (j & 31);
        }
        tail.path[tid][word] = bits;
      }
    }

    // ---- loads of a tile. Block tables, masks and positions come in windows of 64 blocks, a block a lane, two tiles ahead ----
    auto window = [&](const int32_t* rows, int t) {
      return rows[bt_row + min((((t * kTile) >> logP) & ~63) + lane, hot.max_blocks - 1)];
    };
    auto in_window = [&](int t) { return ((t * kTile) >> logP) & 63; };  // the tile's first block in its window
    auto of_slot = [&](int w, int t, int s) { return __builtin_amdgcn_ds_bpermute(4 * (in_window(t) + (s >> logP)), w); };
    auto of_block = [&](int w, int t, int blk) { return __builtin_amdgcn_readlane(w, in_window(t) + blk); };
    auto in_pool = [&](int page) { return (size_t)max(min(page, hot.num_pages - 1), 0); };
    constexpr int kPages = kSlotStep ? kHalves : 1;
    struct Keys { typename std::conditional<kFp8, uint2, uint4>::type lo, hi; };  // eight elements each
    struct Data { Keys k[kHalves]; uint4 v[kVGranules]; };
    auto load_k = [&](Data& d, const int (&page)[kPages]) {
      const int s = sl & (P - 1);
#pragma unroll
      for (int i = 0; i < kHalves; ++i) {
        const unsigned char* pk = kp + in_pool(page[kSlotStep ? i : 0]) * page_bytes;
        const int c = pc + i * kOctetStep;
        if constexpr (kFp8) {  // half a granule
          pk += ((c >> 1) * P + s) * 16 + (c & 1) * 8;
          d.k[i].lo = *reinterpret_cast<const uint2*>(pk);
          d.k[i].hi = *reinterpret_cast<const uint2*>(pk + DX / 2 * P * 16);
        } else {
          pk += (c * P + s) * 16;
          d.k[i].lo = *reinterpret_cast<const uint4*>(pk);
          d.k[i].hi = *reinterpret_cast<const uint4*>(pk + DX / 2 * P * 16);
        }
      }
    };
    auto load_v = [&](Data& d, int page) {
      const unsigned char* pv = vp + in_pool(page) * page_bytes;
#pragma unroll
      for (int i = 0; i < kVGranules; ++i) d.v[i] = *reinterpret_cast<const uint4*>(pv + (uint32_t)((v_first + 64 * i + lane) * 16));
    };

    // ---- queries of the wave's rows ----
    const int base = kWindows ? t0 * kTile : 0;  // positions are counted from here
    Frag q[kTiles][kSteps];
    float turned_q[kWindows ? kSteps : 1][8];
    float row_scale[kTiles];
    int row_node[kTiles];
#pragma unroll
    for (int nr = 0; nr < kTiles; ++nr) {
      const int row = rt * kRows + (rg * kTiles + nr) * 16 + n16, node = row / a.G, head = row - node * a.G;
      const bool there = node < min(r.T, ta.max_q);
      row_node[nr] = there ? min(node, MEPIC_TREE_MAX_NODES - 1) : 0;
      float x[kSteps][8];
      const uint16_t* src = static_cast<const uint16_t*>(a.q) + ((size_t)(r.q0 + row_node[nr]) * a.Hq + (size_t)hk * a.G + head) * D;
      const float pos = there ? (float)(int)((uint32_t)a.q_positions[r.q0 + row_node[nr]] - (uint32_t)base) : 0.f;
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (there) __builtin_memcpy(&u, src + 8 * (4 * kk + g), 16);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          x[kk][2 * j] = __uint_as_float(w[j] << 16);
          x[kk][2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        }
      }
      auto turned = [&](float& lo, float& hi, int i) {
        const float f = turns_frac(pos, a.freq_hi[i], a.freq_lo[i]);
        const float c = __builtin_amdgcn_cosf(f), s = __builtin_amdgcn_sinf(f);
        const float y = lo * c - hi * s;
        hi = hi * c + lo * s;
        lo = y;
      };
      float most = 0.f;
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (inter) {
            if (j % 2 == 0) turned(x[kk][j], x[kk][j + 1], 4 * (4 * kk + g) + j / 2);
          } else {
            if (kk < kSteps / 2) turned(x[kk][j], x[kk + kSteps / 2][j], 8 * (4 * kk + g) + j);
          }
        }
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[kk][j]));
      most = max_over_kgroups(most);
      const int e = most > 0.f ? max(__builtin_amdgcn_frexp_expf(most), -100) : 0;
      row_scale[nr] = ldexpf(a.qk_scale_log2 / kKeyFactor, e);
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float u = ldexpf(x[kk][2 * j], -e), w = ldexpf(x[kk][2 * j + 1], -e);
          q[nr][kk].w[j] = pack2_f16(u, w);
          if constexpr (kWindows) {
            turned_q[kk][2 * j] = u;
            turned_q[kk][2 * j + 1] = w;
          }
        }
    }
    auto next_window = [&]() {  // the queries as seen from 2 kTile positions further on
#pragma unroll
      for (int kk = 0; kk < kSteps / 2; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float2 w = tail.back[8 * (4 * kk + g) + j];
          float &lo = turned_q[kk][j], &hi = turned_q[kk + kSteps / 2][j];
          const float y = lo * w.x + hi * w.y;
          hi = hi * w.x - lo * w.y;
          lo = y;
        }
#pragma unroll
      for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
        for (int j = 0; j < 4; ++j) q[0][kk].w[j] = pack2_f16(turned_q[kk][2 * j], turned_q[kk][2 * j + 1]);
    };
    if (kWindows && !win_kept) keep_window();

    floatx4 o[kTiles][kDims], ones[kTiles];  // ones: products of P with ones, i.e. sums of the weights (bf16 pages)
    float top[kTiles], ref[kTiles], sum[kTiles], least[kTiles];  // reference maximum, the same or 0, sum of weights, least score
#pragma unroll
    for (int nr = 0; nr < kTiles; ++nr) {
      top[nr] = -INFINITY;
      ref[nr] = sum[nr] = 0.f;
      least[nr] = INFINITY;
      ones[nr] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < kDims; ++dt) o[nr][dt] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const bool busy = (rg * kTiles) * 16 < n_rows;  // does the wave have rows?

    float cs[kSets][8], sn[kSets][8];
    int pos_now = 0;
    Data d;
    const int32_t* masks = kPlain || !hot.block_valid_mask ? nullptr : reinterpret_cast<const int32_t*>(hot.block_valid_mask);
    const int32_t* starts = kPlain ? nullptr : hot.block_positions;
    int mask = masks ? window(masks, t0) : -1, start = starts ? window(starts, t0) : 0;  // of tile t, then of the next one
    const int second = min(t0 + 1, t1 - 1);
    int pages = window(hot.block_tables, t0), mask1 = masks ? window(masks, second) : -1, start1 = starts ? window(starts, second) : 0;
    int k_page[kPages], v_from;
    float k_scale = 0.f, v_scale = 0.f;
    // page ids of tile t for its loads, and its scales; then on to the window of tile `after`
    auto take_pages = [&](int t, int after) {
#pragma unroll
      for (int i = 0; i < kPages; ++i) k_page[i] = of_slot(pages, t, sl + i * kSlotStep);
      v_from = of_block(pages, t, v_page);
      if constexpr (kFp8) {
        k_scale = hot.k_scales[in_pool(pages)];
        v_scale = hot.v_scales[in_pool(pages)];
      }
      pages = window(hot.block_tables, after);
    };
    take_pages(t0, second);
    load_k(d, k_page);
    load_v(d, v_from);

    int mask_used = -1;  // what the products of the last staged tile need
    float ks_used = 0.f, vs_used = 0.f;
    auto stage = [&](auto odd, int t) {  // tile t (the second one of its window if odd) into its buffer, and the loads of tile t + 1
      unsigned char* buf = lds + (t & 1) * kTileBytes;
      const int first = t * kTile, slots_left = r.kv_len - first;
      const bool has_nodes = first + kTile > r.ctx;
      const bool fresh = ((t - t0) & (kReseed - 1)) == 0;
      bool on = false;
      // (loads always, the last tile's are its own again: a wait for some of them has to hold on every path. Ids, masks and scales come first:
      // the next stage needs them first, and loads return in order. Their exchange behind the writes to LDS would wait for those.)
      const int t2 = min(t + 1, t1 - 1), t3 = min(t + 2, t1 - 1);
      mask_used = mask;
      const int start_used = start;
      ks_used = k_scale;
      vs_used = v_scale;
      mask = mask1;
      start = start1;
      take_pages(t2, t3);
      if (masks) mask1 = window(masks, t3);
      if (starts) start1 = window(starts, t3);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < kHalves; ++i) {
        const int s = sl + i * kSlotStep, n = first + s, set = kOctetStep ? i : 0;
        Frag lo, hi;
        if constexpr (kWindows) {
          f16x2 (&c)[4] = win_c[decltype(odd)::value * kHalves + i], (&sn2)[4] = win_s[decltype(odd)::value * kHalves + i];
          if (has_nodes) {  // slots of nodes stand anywhere
            asm volatile("");
            const int seen = first - decltype(odd)::value * kTile;  // where the window begins
            const int pos = n < r.ctx ? n - seen : (int)((uint32_t)tail.node_pos[(n - r.ctx) & (MEPIC_TREE_MAX_NODES - 1)] - (uint32_t)seen);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int i0 = freq_index(set, 2 * j), i1 = freq_index(set, 2 * j + 1);
              const float f0 = turns_frac((float)pos, a.freq_hi[i0], a.freq_lo[i0]), f1 = turns_frac((float)pos, a.freq_hi[i1], a.freq_lo[i1]);
              c[j] = __builtin_bit_cast(f16x2, pack2_f16(__builtin_amdgcn_cosf(f0), __builtin_amdgcn_cosf(f1)));
              sn2[j] = __builtin_bit_cast(f16x2, pack2_f16(__builtin_amdgcn_sinf(f0), __builtin_amdgcn_sinf(f1)));
            }
            win_kept = false;
          }
          uint32_t x[8];  // low dims, high dims
          if constexpr (kFp8) {
            const uint32_t w[4] = {d.k[i].lo.x, d.k[i].lo.y, d.k[i].hi.x, d.k[i].hi.y};
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = f16_of_e4m3(w[j >> 1], j & 1);
          } else {
            const uint32_t w[8] = {d.k[i].lo.x, d.k[i].lo.y, d.k[i].lo.z, d.k[i].lo.w, d.k[i].hi.x, d.k[i].hi.y, d.k[i].hi.z, d.k[i].hi.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = pack2_f16(__uint_as_float(w[j] << 16), __uint_as_float(w[j] & 0xffff0000u));
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const f16x2 u = __builtin_bit_cast(f16x2, x[j]), w = __builtin_bit_cast(f16x2, x[4 + j]);
            lo.w[j] = __builtin_bit_cast(uint32_t, u * c[j] - w * sn2[j]);
            hi.w[j] = __builtin_bit_cast(uint32_t, w * c[j] + u * sn2[j]);
          }
        } else {
          if (!kOctetStep || i == 0) {
            int pos = n;
            if (starts) pos = of_slot(start_used, t, s) + (s & (P - 1));
            if (has_nodes) {
              if (n >= r.ctx) pos = tail.node_pos[(n - r.ctx) & (MEPIC_TREE_MAX_NODES - 1)];
              if (n >= r.kv_len) pos = pos_now + kTurn;
            }
            on = !(fresh && i == 0);
            if (starts || has_nodes) on = on && __all(pos == pos_now + kTurn);
            pos_now = pos;
          }
          float (&c)[8] = cs[set], (&s2)[8] = sn[set];
          if (on) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float y = s2[e] * turn_s[set][e];  // (in this order in place: no register is copied)
              s2[e] *= turn_c[set][e];
              s2[e] = __builtin_fmaf(c[e], turn_s[set][e], s2[e]);
              c[e] = __builtin_fmaf(c[e], turn_c[set][e], -y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const int j = freq_index(set, e);
              const float f = turns_frac((float)pos_now, a.freq_hi[j], a.freq_lo[j]);
              c[e] = kKeyFactor * __builtin_amdgcn_cosf(f);
              s2[e] = kKeyFactor * __builtin_amdgcn_sinf(f);
            }
          }
          float x[16];  // low dims, high dims
          if constexpr (kFp8) {
            const uint32_t w[4] = {d.k[i].lo.x, d.k[i].lo.y, d.k[i].hi.x, d.k[i].hi.y};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const f32x2 p0 = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], false), p1 = __builtin_amdgcn_cvt_pk_f32_fp8(w[j], true);
              x[4 * j] = p0[0]; x[4 * j + 1] = p0[1]; x[4 * j + 2] = p1[0]; x[4 * j + 3] = p1[1];
            }
          } else {
            const uint32_t w[8] = {d.k[i].lo.x, d.k[i].lo.y, d.k[i].lo.z, d.k[i].lo.w, d.k[i].hi.x, d.k[i].hi.y, d.k[i].hi.z, d.k[i].hi.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              x[2 * j] = __uint_as_float(w[j] << 16);
              x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            }
          }
          if (inter) {  // pairs are neighbours: four of the low dims, four of the high ones
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float y = x[2 * e] * c[e] - x[2 * e + 1] * s2[e];
              x[2 * e + 1] = x[2 * e + 1] * c[e] + x[2 * e] * s2[e];
              x[2 * e] = y;
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float y = x[e] * c[e] - x[8 + e] * s2[e];
              x[8 + e] = x[8 + e] * c[e] + x[e] * s2[e];
              x[e] = y;
            }
          }
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            lo.w[j] = pack2_f16(x[2 * j], x[2 * j + 1]);
            hi.w[j] = pack2_f16(x[8 + 2 * j], x[9 + 2 * j]);
          }
        }
        bool live = n < r.kv_len;
        if (masks) {
          const int valid = of_slot(mask_used, t, s);  // (every lane takes part in the exchange)
          live = live && ((valid >> (s & (P - 1))) & 1);
        }
        if (masks ? !__all(live) : slots_left < kTile) {  // slots that take no part may hold anything
          asm volatile("");  // (a branch, not eight selects in every tile)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            lo.w[j] = live ? lo.w[j] : 0u;
            hi.w[j] = live ? hi.w[j] : 0u;
          }
        }
        unsigned char* dst = buf + ((pc + i * kOctetStep) * kTile + place + i * kSlotStep) * 16;
        *reinterpret_cast<uint4*>(dst) = lo.u;
        *reinterpret_cast<uint4*>(dst + D / 16 * kTile * 16) = hi.u;
        __builtin_amdgcn_sched_barrier(0);  // (one slot's widened keys in registers at a time)
      }
      load_k(d, k_page);
      const int v_slot = v_page << logP;
      uint32_t v_bits = low_bits(slots_left - v_slot);  // of the page's slots those that take part
      if (masks) v_bits &= (uint32_t)of_block(mask_used, t, v_page);
      const bool v_whole = (v_bits | ~low_bits(P)) == ~0u;
#pragma unroll
      for (int i = 0; i < kVGranules; ++i) {
        Frag f[X / 8];
        if constexpr (kFp8) {
          const uint32_t w[4] = {d.v[i].x, d.v[i].y, d.v[i].z, d.v[i].w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            f[j / 2].w[2 * (j & 1)] = f16_of_e4m3(w[j], false);
            f[j / 2].w[2 * (j & 1) + 1] = f16_of_e4m3(w[j], true);
          }
        } else {
          f[0].u = d.v[i];
        }
#pragma unroll
        for (int h = 0; h < X / 8; ++h) {
          if (!v_whole) {
            asm volatile("");
            const uint32_t keep = v_bits >> (8 * (v_part * (X / 8) + h));
#pragma unroll
            for (int j = 0; j < 4; ++j)
              f[h].w[j] &= ((keep >> (2 * j)) & 1u ? 0x0000ffffu : 0u) | ((keep >> (2 * j + 1)) & 1u ? 0xffff0000u : 0u);
          }
          *reinterpret_cast<uint4*>(buf + v_dst[h] + i * v_stride) = f[h].u;
        }
      }
      load_v(d, v_from);
    };
    auto products = [&](int t, int mask0, float ks0, float vs0) {
      const unsigned char* buf = lds + (t & 1) * kTileBytes;
      const int first = t * kTile, slots_left = r.kv_len - first;
#pragma unroll 1
      for (int sub = 0; sub < kSubs; ++sub) {
        const int grp = sg * kSubs + sub, n0 = first + 32 * grp;
        floatx4 s[kTiles][2];
#pragma unroll
        for (int nr = 0; nr < kTiles; ++nr) s[nr][0] = s[nr][1] = floatx4{0.f, 0.f, 0.f, 0.f};
        // Operands come through a ring of kRing registers sets, each read right behind the product that frees its place; the order is
        // pinned (left to itself the compiler waits for each read before it requests the next).
        Frag k[kRing];
        auto k_at = [&](int i) { return *reinterpret_cast<const uint4*>(buf + k_src + grp * 512 + (4 * (i >> 1) * kTile + 16 * (i & 1)) * 16); };
#pragma unroll
        for (int i = 0; i < kRing; ++i) k[i].u = k_at(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 2 * kSteps; ++i) {
#pragma unroll
          for (int nr = 0; nr < kTiles; ++nr) s[nr][i & 1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[i % kRing].hv, q[nr][i >> 1].hv, s[nr][i & 1], 0, 0, 0);
          if (i + kRing < 2 * kSteps) {
            k[i % kRing].u = k_at(i + kRing);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        Frag v[kRing];
        auto v_at = [&](int dt) { return *reinterpret_cast<const uint4*>(buf + v_src + grp * (4 * D * 16) + dt * 256); };
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kRing && i < kDims; ++i) v[i].u = v_at(i);
        __builtin_amdgcn_sched_barrier(0);
        uint32_t word = low_bits(slots_left - 32 * grp);  // slots that take part
        if (masks)
          word &= P == 32 ? (uint32_t)of_block(mask0, t, grp)
                          : ((uint32_t)of_block(mask0, t, 2 * grp) & 0xffffu) | ((uint32_t)of_block(mask0, t, 2 * grp + 1) << 16);
        const bool some = word != ~0u || n0 + 32 > r.ctx;
        float ks = 1.f, ve = 0.f, vm = 1.f, vi = 1.f;  // K scale, V scale = 2^ve vm, vi = 2^-ve
        if constexpr (kFp8) {
          auto of = [&](float w, int blk) { return __uint_as_float((uint32_t)of_block((int)__float_as_uint(w), t, blk)); };
          float vs;
          if (P == 32) {
            ks = of(ks0, grp);
            vs = of(vs0, grp);
          } else {
            const float k0 = of(ks0, 2 * grp), k1 = of(ks0, 2 * grp + 1), v0 = of(vs0, 2 * grp), v1 = of(vs0, 2 * grp + 1);
            ks = g < 2 ? k0 : k1;
            vs = g < 2 ? v0 : v1;
          }
          // (pages none of whose slots takes part may have any scale; a K scale of 0 would make NaN of the scores masked below)
          const bool used = ((word >> (P == 32 ? 0 : 16 * (g >> 1))) & low_bits(P)) != 0;
          ks = !used ? 1.f : ks == 0.f ? 1e-30f : ks;
          vs = used ? vs : 0.f;
          const int e = min(max(__builtin_amdgcn_frexp_expf(vs), -100), 100);
          ve = (float)e;
          vm = ldexpf(vs, -e);
          vi = ldexpf(1.f, -e);
        }
        Frag p[kTiles];
#pragma unroll
        for (int nr = 0; nr < kTiles; ++nr) {
          float y[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) y[j] = s[nr][j >> 2][j & 3];
          if constexpr (!kFp8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) least[nr] = fminf(least[nr], y[j]);
          }
          if (some) {
            const uint32_t bits = (word & path_bits(tail.path[row_node[nr]], n0, r.ctx)) >> (8 * g);
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = (bits >> j) & 1u ? y[j] : -INFINITY;
          }
          const float c = row_scale[nr] * ks;
          float most = y[0];
#pragma unroll
          for (int j = 1; j < 8; ++j) most = fmaxf(most, y[j]);
          most = most == -INFINITY ? most : __builtin_fmaf(most, c, ve);
          if (__any(most > top[nr] + 8.f)) {
            const float now_top = fmaxf(top[nr], max_over_kgroups(most));
            const float f = now_top == top[nr] ? 1.f : __builtin_amdgcn_exp2f(top[nr] - now_top);
            top[nr] = now_top;
            ref[nr] = now_top == -INFINITY ? 0.f : now_top;
            sum[nr] *= f;
#pragma unroll
            for (int i = 0; i < 4; ++i) ones[nr][i] *= f;
#pragma unroll
            for (int dt = 0; dt < kDims; ++dt)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[nr][dt][i] *= f;
          }
          const float shift = ve - ref[nr];
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(y[j], c, shift));
            if (kFp8) part += y[j];
          }
          if constexpr (kFp8) {
            sum[nr] = __builtin_fmaf(part, vi, sum[nr]);
#pragma unroll
            for (int j = 0; j < 4; ++j) p[nr].w[j] = pack2_f16(y[2 * j] * vm, y[2 * j + 1] * vm);
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) p[nr].w[j] = pack2_bf16(y[2 * j], y[2 * j + 1]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kFp8) {
          Frag one;
          one.w[0] = one.w[1] = one.w[2] = one.w[3] = 0x3f803f80u;
#pragma unroll
          for (int nr = 0; nr < kTiles; ++nr) ones[nr] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(one.v, p[nr].v, ones[nr], 0, 0, 0);
        }
#pragma unroll
        for (int dt = 0; dt < kDims; ++dt) {
#pragma unroll
          for (int nr = 0; nr < kTiles; ++nr) {
            if constexpr (kFp8) o[nr][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v[dt % kRing].hv, p[nr].hv, o[nr][dt], 0, 0, 0);
            else o[nr][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[dt % kRing].v, p[nr].v, o[nr][dt], 0, 0, 0);
          }
          if (dt + kRing < kDims) {
            v[dt % kRing].u = v_at(dt + kRing);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    };

    constexpr std::integral_constant<int, 0> kEven;
    constexpr std::integral_constant<int, kWindows ? 1 : 0> kOdd;
    // (the loop is entered where the first tile is staged: one copy of the code less, which a short run would fetch for nothing)
#pragma unroll 1
    for (int t = t0 - 1;;) {
      if (busy && t >= t0) products(t, mask_used, ks_used, vs_used);
      if (t + 1 < t1) stage(kEven, t + 1);
      __syncthreads();
      if (++t == t1) break;
      if constexpr (kWindows) {
        if (busy) {
          if (t > t0) next_window();
          products(t, mask_used, ks_used, vs_used);
        }
        if (t + 1 < t1) stage(kOdd, t + 1);
        __syncthreads();
        if (++t == t1) break;
      }
    }

    // ---- rows written; where several waves share a row's slots, they are merged first ----
    const int rows_here = min(n_rows, kRows);
    const bool direct = t0 == 0 && t1 == tiles;
    const size_t part = ((size_t)blockIdx.x * 2 + (t0 == 0 ? 1 : 0)) * kRows;
    // four dims of a row: its output, divided by the sum of weights, or its partial
    auto put = [&](int row, int dim, const floatx4& x, float mx, float den, float inv, uint16_t* out) {
      if (direct) {
        uint2 w;
        w.x = pack2_bf16(x[0] * inv, x[1] * inv);
        w.y = pack2_bf16(x[2] * inv, x[3] * inv);
        __builtin_memcpy(out + dim, &w, 8);
      } else {
        *reinterpret_cast<floatx4*>(tail.part_o + (part + row) * D + dim) = x;
        if (dim == 0) *reinterpret_cast<float2*>(tail.part_ml + (part + row) * 2) = make_float2(mx, den);
      }
    };
    auto out_of = [&](int row) {
      const int all = rt * kRows + row, node = all / a.G, head = all - node * a.G;
      return static_cast<uint16_t*>(a.out) + ((size_t)(r.q0 + node) * a.Hq + (size_t)hk * a.G + head) * D;
    };
    auto mark = [&](int row, float odd) {  // odd is NaN if anything is Inf or NaN
      if (direct && !(odd == 0.f)) atomicOr(&tail.bad[row >> 5], 1u << (row & 31));
    };
    if constexpr (kSlotGroups == 1) {
      if (busy) {
#pragma unroll
        for (int nr = 0; nr < kTiles; ++nr) {
          const int row = (wave * kTiles + nr) * 16 + n16;
          const float total_w = kFp8 ? sum_over_kgroups(sum[nr]) : ones[nr][0];
          const float den = -max_over_kgroups(-least[nr]) == -INFINITY ? NAN : total_w;
          if (row < rows_here) {
            const bool none = top[nr] == -INFINITY && den == 0.f;  // no slot took part
            const float inv = den != 0.f ? 1.f / den : 0.f;
            uint16_t* out = out_of(row);
            float odd = den * 0.f;
#pragma unroll
            for (int dt = 0; dt < kDims; ++dt) {
              const floatx4 x = none ? floatx4{0.f, 0.f, 0.f, 0.f} : o[nr][dt];
              odd += (x[0] + x[1] + x[2] + x[3]) * 0.f;
              put(row, 16 * dt + 4 * g, x, top[nr], den, inv, out);
            }
            mark(row, odd);
          }
        }
      }
    } else {
      if (busy) {
#pragma unroll
        for (int nr = 0; nr < kTiles; ++nr) {
          const float total_w = kFp8 ? sum_over_kgroups(sum[nr]) : ones[nr][0];
          const float low = -max_over_kgroups(-least[nr]);
          const int row = nr * 16 + n16;
          if (g == 0) {
            tail.ml[wave][row][0] = top[nr];
            tail.ml[wave][row][1] = low == -INFINITY ? NAN : total_w;
          }
          float* dst = reinterpret_cast<float*>(lds) + (size_t)(wave * kTiles * 16 + row) * D;
#pragma unroll
          for (int dt = 0; dt < kDims; ++dt) *reinterpret_cast<floatx4*>(dst + 4 * ((4 * dt + g) ^ n16)) = o[nr][dt];
        }
      }
      __syncthreads();
      constexpr int kQuads = D / 4;
      for (int u = tid; u < rows_here * kQuads; u += kThreads) {
        const int row = u / kQuads, quad = u % kQuads, in = row % (16 * kTiles), w0 = row / (16 * kTiles);
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < kSlotGroups; ++i) mx = fmaxf(mx, tail.ml[w0 + i * kGroups][in][0]);
        float den = 0.f;
        floatx4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kSlotGroups; ++i) {
          const int w = w0 + i * kGroups;
          const float mi = tail.ml[w][in][0], li = tail.ml[w][in][1];
          if (mi == -INFINITY && li == 0.f) continue;  // no slot took part
          const float f = mi == mx ? 1.f : __builtin_amdgcn_exp2f(mi - mx);
          const floatx4 y = *reinterpret_cast<const floatx4*>(reinterpret_cast<const float*>(lds) + (size_t)(w * kTiles * 16 + in) * D + 4 * (quad ^ (in & 15)));
          den += f * li;
#pragma unroll
          for (int j = 0; j < 4; ++j) x[j] += f * y[j];
        }
        put(row, 4 * quad, x, mx, den, den != 0.f ? 1.f / den : 0.f, out_of(row));
        mark(row, (x[0] + x[1] + x[2] + x[3]) * 0.f + den * 0.f);
      }
    }
    __syncthreads();
    for (int w = 0; direct && w < kRows / 32; ++w) {
      const uint32_t all_bits = uni(tail.bad[w]);
      for (uint32_t bits = all_bits; bits; bits &= bits - 1) {
        const int all = rt * kRows + 32 * w + __builtin_ctz(bits), node = all / a.G, head = all - node * a.G;
        tree_row<kFp8 ? MEPIC_F8E4M3 : MEPIC_BF16, kThreads>(ta, tail.row, r, b, node, hk * a.G + head);
      }
      if (all_bits && tid == 0) tail.bad[w] = 0;  // (tree_row has barriers: every wave has read it)
    }
  }
}

}  // namespace mepic
