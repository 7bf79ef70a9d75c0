// Attention of a tree of drafted tokens on the matrix cores, e4m3 pages: the kernels of tree_tiles.h for every size of row tile.
#include "split_common.h"
#include "tree_tiles.h"

namespace mepic {
namespace {

template <int D, int kWaves, int kGroups, int kTiles, bool kPlain>
hipError_t launch_one(const TreeMfmaArgs& m, hipStream_t s) {
  static std::atomic<uint64_t> asked{0};
  const auto kernel = tree_tiles_kernel<true, D, kWaves, kGroups, kTiles, kPlain>;
  constexpr size_t bytes = tree_lds_bytes<D, kWaves>();
  const hipError_t e = allow_lds(reinterpret_cast<const void*>(kernel), bytes, asked);
  if (e != hipSuccess) return e;
  kernel<<<dim3((unsigned)m.groups * m.t.a.Hkv), dim3(kWaves * 64), bytes, s>>>(m);
  return hipGetLastError();
}

template <int D, bool kPlain>
hipError_t launch_rows(int rows, const TreeMfmaArgs& m, hipStream_t s) {
  if (rows == 32) return launch_one<D, 8, 2, 1, kPlain>(m, s);
  if (rows == 64) return launch_one<D, 4, 4, 1, kPlain>(m, s);
  if (rows == 128) return launch_one<D, 4, 4, 2, kPlain>(m, s);
  if (rows == 256) return launch_one<D, 8, 8, 2, kPlain>(m, s);
  return hipErrorInvalidValue;  // (a plan for other rows has a workspace of other sizes)
}

}  // namespace

hipError_t launch_tree_tiles_fp8(int rows, const TreeMfmaArgs& m, hipStream_t s) {
  const bool plain = !m.t.a.interleaved && !m.t.a.block_positions && !m.t.a.block_valid_mask;
  if (m.t.a.D == 128) return plain ? launch_rows<128, true>(rows, m, s) : launch_rows<128, false>(rows, m, s);
  return plain ? launch_rows<64, true>(rows, m, s) : launch_rows<64, false>(rows, m, s);
}

}  // namespace mepic
