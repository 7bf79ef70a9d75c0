// Keep one path of a tree of drafted tokens (§3.3.2): the K/V of the accepted nodes, scattered over the slots behind the context, move
// to the first of them, in place. The r-th kept node k_r (ascending) goes from slot first + k_r to first + r <= first + k_r, which lies
// before the source of every later node: tokens may be moved in ascending order, a group of them read before any of it is written.
//
// One workgroup per (request, KV head) takes groups of kGroup tokens: slots and pages of the group are resolved into LDS, all its
// granules of K and elements of V are requested, and after a barrier stored. Bound by the chain of dependent loads (prefix sums,
// node, block table, scale, K/V), each some 2 us with what starts and ends a launch: the bytes are few. Measured: 64 requests with 26 drafted tokens
// at most 16.3 - 17.5 us, 1024 with 64 on e4m3 pages 21.2. Lanes across the dims of one token leave whole waves out of tokens that are not
// there; across the tokens of one dim, whose elements of V are neighbours, the same calls take 17.6 and 26.3.
#include "attn_common.h"

namespace mepic {
namespace {

constexpr int kThreads = 256, kGroup = 16;

struct KeepArgs {
  void* k_pages;
  void* v_pages;
  const float* k_scales;
  const float* v_scales;
  const int32_t* block_tables;
  const int32_t* first_slots;
  const int32_t* cu_tree;
  const int32_t* kept;
  const int32_t* cu_kept;
  int32_t* kv_lens_out;
  int32_t B, n_kept, Hkv, max_blocks, num_pages;
};

struct alignas(16) Granule { uint32_t w[4]; };

// Four e4m3 codes of a page with scale `from` as codes of a page with scale `to`, rounded as the commit step rounds.
__device__ __forceinline__ uint32_t requant4(uint32_t codes, float from, float to) {
  float y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const f32x2 x = e < 2 ? __builtin_amdgcn_cvt_pk_f32_fp8(codes, false) : __builtin_amdgcn_cvt_pk_f32_fp8(codes, true);
    y[e] = __builtin_fminf(__builtin_fmaxf(x[e & 1] * from / to, -448.f), 448.f);
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (uint32_t)w;
}

template <typename T, int D, int P>
__global__ __launch_bounds__(kThreads) void kv_keep_kernel(const KeepArgs a) {
  constexpr int X = 16 / (int)sizeof(T), DX = D / X;
  constexpr bool kFp8 = sizeof(T) == 1;
  constexpr int kUnitsK = (kGroup * DX + kThreads - 1) / kThreads, kUnitsV = (kGroup * D + kThreads - 1) / kThreads;
  __shared__ int s_from_page[kGroup], s_from[kGroup], s_to_page[kGroup], s_to[kGroup];  // page -1: nothing to move
  __shared__ float s_scale[kGroup][4];  // K from, K to, V from, V to
  const int b = blockIdx.x, h = blockIdx.y, tid = threadIdx.x;
  const int first = a.first_slots[b];
  if (first < 0) return;
  const int nodes = a.cu_tree[b + 1] - a.cu_tree[b];
  const int k0 = max(a.cu_kept[b], 0), count = max(min(a.cu_kept[b + 1], a.n_kept) - k0, 0);
  if (h == 0 && tid == 0 && a.kv_lens_out) a.kv_lens_out[b] = first + count;
  T* kp = static_cast<T*>(a.k_pages);
  T* vp = static_cast<T*>(a.v_pages);
  for (int r0 = 0; r0 < count; r0 += kGroup) {
    if (tid < kGroup) {
      const int r = r0 + tid;
      int from_page = -1, to_page = -1, from = 0, to = 0;
      if (r < count) {
        const int node = a.kept[k0 + r];
        const bool rises = r == 0 || node > a.kept[k0 + r - 1];
        const long nf = (long)first + node, nt = (long)first + r;
        if (rises && node > r && node < nodes && nf / P < a.max_blocks) {  // (node == r: it lies where it belongs)
          const int pf = a.block_tables[(long)b * a.max_blocks + nf / P], pt = a.block_tables[(long)b * a.max_blocks + nt / P];
          if (pf >= 0 && pf < a.num_pages && pt >= 0 && pt < a.num_pages) {
            from_page = pf; to_page = pt;
            from = (int)(nf % P); to = (int)(nt % P);
            if constexpr (kFp8) {
              s_scale[tid][0] = a.k_scales[pf]; s_scale[tid][1] = a.k_scales[pt];
              s_scale[tid][2] = a.v_scales[pf]; s_scale[tid][3] = a.v_scales[pt];
            }
          }
        }
      }
      s_from_page[tid] = from_page; s_to_page[tid] = to_page; s_from[tid] = from; s_to[tid] = to;
    }
    __syncthreads();
    Granule k[kUnitsK];
    T v[kUnitsV];
#pragma unroll
    for (int j = 0; j < kUnitsK; ++j) {
      const int u = tid + j * kThreads, i = u / DX, dc = u % DX;
      if (i < kGroup && s_from_page[i] >= 0)
        k[j] = *reinterpret_cast<const Granule*>(kp + ((((size_t)s_from_page[i] * a.Hkv + h) * DX + dc) * P + s_from[i]) * X);
    }
#pragma unroll
    for (int j = 0; j < kUnitsV; ++j) {
      const int u = tid + j * kThreads, i = u / D, d = u % D;
      if (i < kGroup && s_from_page[i] >= 0) v[j] = vp[(((size_t)s_from_page[i] * a.Hkv + h) * D + d) * P + s_from[i]];
    }
    __syncthreads();  // the group is read whole
#pragma unroll
    for (int j = 0; j < kUnitsK; ++j) {
      const int u = tid + j * kThreads, i = u / DX, dc = u % DX;
      if (i >= kGroup || s_from_page[i] < 0) continue;
      if constexpr (kFp8) {
        if (s_scale[i][0] != s_scale[i][1])
#pragma unroll
          for (int e = 0; e < 4; ++e) k[j].w[e] = requant4(k[j].w[e], s_scale[i][0], s_scale[i][1]);
      }
      *reinterpret_cast<Granule*>(kp + ((((size_t)s_to_page[i] * a.Hkv + h) * DX + dc) * P + s_to[i]) * X) = k[j];
    }
#pragma unroll
    for (int j = 0; j < kUnitsV; ++j) {
      const int u = tid + j * kThreads, i = u / D, d = u % D;
      if (i >= kGroup || s_from_page[i] < 0) continue;
      T x = v[j];
      if constexpr (kFp8) {
        if (s_scale[i][2] != s_scale[i][3]) x = (T)(requant4(x, s_scale[i][2], s_scale[i][3]) & 0xffu);
      }
      vp[(((size_t)s_to_page[i] * a.Hkv + h) * D + d) * P + s_to[i]] = x;
    }
    __syncthreads();  // the group is written, its slots may be resolved anew
  }
}

template <typename T>
hipError_t launch(const KeepArgs& a, int D, int P, hipStream_t s) {
  const dim3 grid(a.B, a.Hkv);
  if (D == 128 && P == 16) kv_keep_kernel<T, 128, 16><<<grid, kThreads, 0, s>>>(a);
  else if (D == 128) kv_keep_kernel<T, 128, 32><<<grid, kThreads, 0, s>>>(a);
  else if (P == 16) kv_keep_kernel<T, 64, 16><<<grid, kThreads, 0, s>>>(a);
  else kv_keep_kernel<T, 64, 32><<<grid, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace
}  // namespace mepic

extern "C" int mepic_kv_keep(const mepic_keep_params* p, void* hip_stream) {
  using namespace mepic;
  if (!p) return MEPIC_ERR_INVALID;
  if (p->B < 0 || p->n_kept < 0 || p->Hkv <= 0 || p->max_blocks < 0 || p->num_pages < 0) return MEPIC_ERR_INVALID;
  if (p->kv_dtype != MEPIC_F32 && p->kv_dtype != MEPIC_BF16 && p->kv_dtype != MEPIC_F8E4M3) return MEPIC_ERR_UNSUPPORTED;
  if ((p->D != 64 && p->D != 128) || (p->P != 16 && p->P != 32) || p->Hkv > 65535) return MEPIC_ERR_UNSUPPORTED;
  if (p->B == 0) return MEPIC_OK;
  if (!p->k_pages || !p->v_pages || !p->block_tables || !p->first_slots || !p->cu_tree || !p->cu_kept || (p->n_kept && !p->kept))
    return MEPIC_ERR_INVALID;
  if (p->kv_dtype == MEPIC_F8E4M3 && (!p->k_scales || !p->v_scales)) return MEPIC_ERR_INVALID;
  const KeepArgs a{p->k_pages, p->v_pages, p->k_scales, p->v_scales, p->block_tables, p->first_slots, p->cu_tree, p->kept, p->cu_kept,
                   p->kv_lens_out, p->B, p->n_kept, p->Hkv, p->max_blocks, p->num_pages};
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  hipError_t e;
  if (p->kv_dtype == MEPIC_F8E4M3) e = launch<uint8_t>(a, p->D, p->P, s);
  else if (p->kv_dtype == MEPIC_BF16) e = launch<uint16_t>(a, p->D, p->P, s);
  else e = launch<float>(a, p->D, p->P, s);
  return e == hipSuccess ? MEPIC_OK : MEPIC_ERR_LAUNCH;
}
