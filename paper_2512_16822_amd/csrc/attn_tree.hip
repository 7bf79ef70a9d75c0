// Attention of a tree of drafted tokens, general form: every case the call allows, in plain fp32 arithmetic. One workgroup per output
// row; it is what the matrix-core kernels fall back to for rows that came out Inf or NaN.
#include "tree_common.h"

namespace mepic {
namespace {

constexpr int kRowThreads = 256;

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

}  // namespace

hipError_t launch_tree_general(const TreeArgs& t, hipStream_t s) {
  const dim3 grid((unsigned)t.a.n_q * t.a.Hq);
  if (t.a.kv_dtype == MEPIC_F32) tree_general_kernel<MEPIC_F32><<<grid, kRowThreads, 0, s>>>(t);
  else if (t.a.kv_dtype == MEPIC_BF16) tree_general_kernel<MEPIC_BF16><<<grid, kRowThreads, 0, s>>>(t);
  else tree_general_kernel<MEPIC_F8E4M3><<<grid, kRowThreads, 0, s>>>(t);
  return hipGetLastError();
}

}  // namespace mepic
