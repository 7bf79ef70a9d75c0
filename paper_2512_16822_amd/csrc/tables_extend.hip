// Block tables, slot maps and positions of the tokens a step appends (§3.2.3), from lengths on the device.
//
// One workgroup scans the requests: how many pages each needs and how many tokens it brings, as inclusive prefix sums over chunks of
// kThreads requests (lane shifts inside a wave, one exchange between waves). Demand only grows along the prefix, so "served" is a
// comparison per request: demand up to and with it against what the list holds. Then every new block and every token finds its request by binary
// search in the prefix sums. Bound by launches and the chain of dependent loads; the bytes are few (272 requests of up to 4 K new tokens, 12 MB:
// 17.4 us, of which the first launch is 5.4). A call of no more tokens than that workgroup has threads does the second part in it too:
// us a call in one and in two launches, 770 tokens of 16 requests 8.1 and 9.7, 900 of 64 8.6 and 9.6; 1500 of 512 12.2 and 10.8, 2100 of 64 12.0 and 10.4.
#include <climits>

#include "attn_common.h"

namespace mepic {
namespace {

constexpr int kThreads = 1024;

struct ExtendArgs {
  mepic_extend_params p;
  int32_t* first_page;  // workspace [B+1]: pages asked for before each request
  int32_t* held;        // workspace [B+1]: blocks that had a page; [B]: entries of the list used before
};

// Inclusive prefix sum over the workgroup, `carry` in front; every thread gets its own, and carry becomes the total (at most
// 2^31 requests of 2^31 each).
__device__ __forceinline__ long long scan(long long x, long long& carry, long long* lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  if (lane == 63) lds[wave] = x;
  __syncthreads();
  long long before = carry, total = carry;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) {
    if (w < wave) before += lds[w];
    total += lds[w];
  }
  __syncthreads();
  carry = total;
  return x + before;
}

__device__ __forceinline__ int32_t fit(long long x) { return x > INT_MAX ? INT_MAX : (int32_t)x; }

// The requests' part, by the kThreads threads of one workgroup.
__device__ __forceinline__ void extend_requests(const ExtendArgs& e) {
  const mepic_extend_params& p = e.p;
  __shared__ long long lds[kThreads / 64];
  const bool pages = p.free_head != nullptr;
  const int head = pages ? max(*p.free_head, 0) : 0;
  const long long room = pages ? max(p.n_free - head, 0) : 0;
  long long tokens = 0, demand = 0, served_pages = 0;
  for (int b0 = 0; b0 < p.B; b0 += kThreads) {
    const int b = b0 + threadIdx.x;
    const bool here = b < p.B;
    const int kv = here ? p.kv_lens[b] : 0, add = here ? p.new_lens[b] : 0, held = here && pages ? p.n_blocks[b] : 0;
    const bool bad = kv < 0 || add < 0 || held < 0;
    const int n = bad ? 0 : add;
    const long long len = (long long)kv + n, blocks = (len + p.P - 1) / p.P;
    const bool wide = !bad && blocks <= p.max_blocks && len <= INT_MAX;
    const int need = wide && pages ? max((int)blocks - held, 0) : 0;
    const long long tok = scan(n, tokens, lds), upto = scan(need, demand, lds);
    const bool served = wide && (need == 0 || upto <= room);
    (void)scan(served ? need : 0, served_pages, lds);
    if (here) {
      p.cu_tokens[b + 1] = fit(tok);
      if (b == 0) p.cu_tokens[0] = 0;
      e.first_page[b] = fit(upto - need);
      e.held[b] = held;
      p.run_request[b] = served ? b : -1;
      p.run_first_slot[b] = served ? kv : -1;
      p.status[b] = bad ? MEPIC_EXTEND_BAD_LENGTH : !wide ? MEPIC_EXTEND_NO_BLOCKS : served ? MEPIC_EXTEND_OK : MEPIC_EXTEND_NO_PAGES;
      p.kv_lens_out[b] = served ? (int)len : kv;
      if (pages) p.n_blocks_out[b] = served ? held + need : held;
    }
  }
  if (threadIdx.x == 0) {
    if (p.B == 0) p.cu_tokens[0] = 0;
    e.first_page[p.B] = fit(demand < room ? demand : room);
    e.held[p.B] = head;
    if (pages) *p.free_head_out = head + (int)served_pages;
  }
}

// Last b with sums[b] <= x, for sums[0] <= x < sums[B].
__device__ __forceinline__ int owner(const int32_t* sums, int B, int x) {
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// The new blocks' and tokens' part: thread `me` of `stride`.
__device__ __forceinline__ void extend_tokens(const ExtendArgs& e, int me, int stride) {
  const mepic_extend_params& p = e.p;
  const int head = e.held[p.B], total = min(p.cu_tokens[p.B], p.max_tokens);
  const bool pages = p.free_head != nullptr;
  if (pages) {
    // (requests that ask for nothing share their first page's number with the next one: the last of them owns it)
    const int wanted = e.first_page[p.B];
    for (int i = me; i < wanted; i += stride) {
      const int b = owner(e.first_page, p.B, i);
      const long long block = (long long)e.held[b] + i - e.first_page[b];
      if (p.run_first_slot[b] >= 0 && block < p.max_blocks) p.block_tables[(size_t)b * p.max_blocks + block] = p.free_pages[head + i];
    }
  }
  for (int t = me; t < total; t += stride) {
    const int b = owner(p.cu_tokens, p.B, t), i = t - p.cu_tokens[b], first = p.run_first_slot[b];
    long long place = -1;
    int pos = -1;
    if (first >= 0) {
      const int n = first + i, block = n / p.P, s = n % p.P, base = p.first_positions ? p.first_positions[b] : first;
      const size_t at = (size_t)b * p.max_blocks + block;
      pos = base + (p.token_offsets ? p.token_offsets[t] : i);
      if (p.token_slots) {
        const int page = pages && block >= e.held[b] ? p.free_pages[head + e.first_page[b] + block - e.held[b]] : p.block_tables[at];
        if (page >= 0 && page < p.num_pages) place = (long long)page * p.P + s;
      }
      if (i == 0 || s == 0) {  // the first of the new tokens in a block writes what the block has once
        if (p.block_positions && s == 0) p.block_positions[at] = base + i;
        if (p.block_valid_mask) {
          const int end = min(p.P, s + p.cu_tokens[b + 1] - t);
          const uint32_t bits = (end < 32 ? (1u << end) - 1u : ~0u) & ~((1u << s) - 1u);
          p.block_valid_mask[at] = s == 0 ? bits : p.block_valid_mask[at] | bits;
        }
      }
    }
    if (p.token_slots) p.token_slots[t] = place;
    if (p.token_positions) p.token_positions[t] = pos;
    if (p.token_requests) p.token_requests[t] = first >= 0 ? b : -1;
  }
}

__global__ __launch_bounds__(kThreads) void extend_requests_kernel(const ExtendArgs e) { extend_requests(e); }

__global__ __launch_bounds__(256) void extend_tokens_kernel(const ExtendArgs e) { extend_tokens(e, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256); }

__global__ __launch_bounds__(kThreads) void extend_small_kernel(const ExtendArgs e) {
  extend_requests(e);
  __syncthreads();  // (what the workgroup has written it may read)
  extend_tokens(e, threadIdx.x, kThreads);
}

int check(const mepic_extend_params* p) {
  if (!p || p->B < 0 || p->max_blocks < 0 || p->num_pages < 0 || p->n_free < 0 || p->max_tokens < 0 || p->P < 1 || p->P > 32)
    return MEPIC_ERR_INVALID;
  return MEPIC_OK;
}

size_t need_bytes(const mepic_extend_params* p) { return 2 * ((size_t)p->B + 1) * sizeof(int32_t); }

}  // namespace
}  // namespace mepic

extern "C" int mepic_tables_extend_workspace_size(const mepic_extend_params* p, size_t* bytes_out) {
  if (!bytes_out) return MEPIC_ERR_INVALID;
  const int rc = mepic::check(p);
  if (rc != MEPIC_OK) return rc;
  *bytes_out = mepic::need_bytes(p);
  return MEPIC_OK;
}

extern "C" int mepic_tables_extend(const mepic_extend_params* p, void* hip_stream) {
  using namespace mepic;
  const int rc = check(p);
  if (rc != MEPIC_OK) return rc;
  if (!p->cu_tokens) return MEPIC_ERR_INVALID;
  if (p->B > 0 && (!p->kv_lens || !p->new_lens || !p->kv_lens_out || !p->run_request || !p->run_first_slot || !p->status ||
                   (p->max_blocks && !p->block_tables)))
    return MEPIC_ERR_INVALID;
  const bool given = p->free_head != nullptr;  // (no request: arrays of no entries may be null)
  if (given != !!p->free_head_out || (p->B > 0 && (given != !!p->n_blocks || given != !!p->n_blocks_out))) return MEPIC_ERR_INVALID;
  if (given ? p->n_free && !p->free_pages : p->free_pages || p->n_free) return MEPIC_ERR_INVALID;
  if (!p->workspace || p->workspace_bytes < need_bytes(p)) return MEPIC_ERR_CAPACITY;
  if (reinterpret_cast<uintptr_t>(p->workspace) & 255u) return MEPIC_ERR_INVALID;
  ExtendArgs e{*p, static_cast<int32_t*>(p->workspace), static_cast<int32_t*>(p->workspace) + p->B + 1};
  hipStream_t s = reinterpret_cast<hipStream_t>(hip_stream);
  const long work = p->max_tokens > 0 ? p->max_tokens : p->n_free;
  if (p->B > 0 && work > 0 && work <= kThreads) {
    extend_small_kernel<<<1, kThreads, 0, s>>>(e);
    return hipGetLastError() == hipSuccess ? MEPIC_OK : MEPIC_ERR_LAUNCH;
  }
  extend_requests_kernel<<<1, kThreads, 0, s>>>(e);
  if (p->B > 0 && work > 0) {
    const long groups = (work + 255) / 256;
    extend_tokens_kernel<<<(unsigned)(groups < 1024 ? groups : 1024), 256, 0, s>>>(e);
  }
  return hipGetLastError() == hipSuccess ? MEPIC_OK : MEPIC_ERR_LAUNCH;
}
