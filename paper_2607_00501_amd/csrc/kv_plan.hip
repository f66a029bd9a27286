// One step's bookkeeping of a batch over a paged KV cache, on the device: the
// pages that the new tokens need come from a ring of free pages, and every new
// token gets its position and its slot (BaseRT Sec. 3.2: all cache memory is
// laid down before the loop starts and nothing is requested in it, so the step
// itself can only hand out pages that exist).
//
// With P tokens a page, request i holding l_i tokens and given t_i new ones:
//   have_i = ceil(l_i / P),  need_i = ceil((l_i + t_i) / P) - have_i,
//   e_i = t_0 + .. + t_i,    u_i = need_0 + .. + need_i  (both inclusive sums),
// page have_i + j of request i is ring entry u_i - need_i + j, and token j of
// request i, at e_i - t_i + j in the batch, has position l_i + j and slot
// page * P + (l_i + j) % P.
//
// Everything follows from three prefix sums over at most 1,024 requests, so the
// whole step is one launch: every workgroup takes the sums over all requests by
// itself (one request a thread, a scan by wavefront and one over the wavefronts)
// and then its own share of the tokens, of the new page table entries and of the
// pages that come back; each finds its request by a binary search in LDS.  What bounds
// it is the chain of those steps and of two dependent loads: 3-5 us for one request,
// 9 for 1,000 with prompts of 30 tokens.  Workgroups of their own for the pages took as long.  What
// a workgroup reads, no other writes: new table entries are not read but taken
// from the ring, pages come back past the ring's last entry.
#include "qm_internal.h"
#include "wave_scan.h"

#include <algorithm>

namespace qm {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanWaves = kPlanThreads / 64;

// Inclusive sum over the workgroup's threads, in thread order.
__device__ __forceinline__ int block_scan(int v, int* wave_sums) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  v = wave_scan(v);
  if (lane == 63) wave_sums[wave] = v;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int w = 0; w < kPlanWaves; ++w) before += w < wave ? wave_sums[w] : 0;
  return v + before;
}

// First i < n with sums[i] > x (sums ascending, sums[n - 1] > x).
__device__ __forceinline__ int first_above(const int* sums, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__global__ __launch_bounds__(kPlanThreads) void kv_plan_kernel(KvPlanArgs a) {
  __shared__ int sums[3][kPlanWaves];
  __shared__ int s_end[kPlanThreads], s_add[kPlanThreads], s_len[kPlanThreads], s_have[kPlanThreads];
  __shared__ int s_upto[kPlanThreads], s_need[kPlanThreads], s_back[kPlanThreads];
  __shared__ int s_taken, s_refused;
  const int i = threadIdx.x, P = 1 << a.page_log2, n = a.n_req;
  if (i == 0) s_taken = s_refused = 0;
  int head = a.ring[0], count = a.ring[1];
  if (head < 0 || head >= a.n_pages || count < 0 || count > a.n_pages) head = count = 0;   // no ring of this size
  int len = 0, t = -1;
  if (i < n) {
    len = a.lens[i];
    t = a.new_lens[i];
  }
  // t < 0: the request has ended.  More new tokens than the batch holds refuse
  // the request whatever their number, so the sums stay below 2^27.
  const bool sane = len >= 0 && len <= static_cast<int64_t>(a.max_pages) << a.page_log2;
  if (sane) len = max(len, a.prefix_pages << a.page_log2);       // the prefix is there from the start
  const int add = i < n ? min(max(t, 0), a.max_tokens + 1) : 0;
  const int end = block_scan(add, sums[0]);
  const bool active = i < n && t >= 0;
  const bool fits = active && sane && static_cast<int64_t>(len) + add <= static_cast<int64_t>(a.max_pages) << a.page_log2 &&
                    end <= a.max_tokens;
  const int have = sane ? (len + P - 1) >> a.page_log2 : 0;
  const int need = fits ? ((len + add + P - 1) >> a.page_log2) - have : 0;
  const int back = i < n && t < 0 && sane ? max(have - a.prefix_pages, 0) : 0;
  const int upto = block_scan(need, sums[1]);
  const int upto_back = block_scan(back, sums[2]);
  const bool granted = fits && (need == 0 || upto <= count);
  s_end[i] = end;
  s_add[i] = add;
  s_len[i] = granted ? len : -1;
  s_have[i] = have;
  s_upto[i] = upto;
  s_need[i] = need;
  s_back[i] = upto_back;
  if (granted && need > 0) atomicMax(&s_taken, upto);
  if (active && !granted) atomicAdd(&s_refused, 1);
  __syncthreads();
  const int taken = s_taken;                                   // the granted ones' pages, in order from the head
  const int given_back = min(s_back[n - 1], a.n_pages - count);
  auto ring_at = [&](int j) __attribute__((always_inline)) {   // 0 <= j < 2 n_pages
    const int64_t at = static_cast<int64_t>(head) + j;
    return static_cast<int>(at % a.n_pages);
  };

  if (blockIdx.x == 0) {
    if (i < n) {
      a.lens_out[i] = active ? (granted ? len + add : len) : sane ? 0 : len;
      a.kv_lens[i] = granted ? len + add : 0;
      a.offsets[i + 1] = min(end, a.max_tokens);
    }
    if (i == 0) {
      a.offsets[0] = 0;
      a.ring_out[0] = ring_at(taken);
      a.ring_out[1] = count - taken + given_back;
      a.refused[0] = s_refused;
    }
  }
  const int first = blockIdx.x * kPlanThreads + i, stride = gridDim.x * kPlanThreads;
  // Tokens.
  const int tokens = min(s_end[n - 1], a.max_tokens);
  for (int x = first; x < a.max_tokens; x += stride) {
    int pos = -1;
    int64_t slot = -1;
    if (x < tokens) {
      const int r = first_above(s_end, n, x);
      if (s_len[r] >= 0) {
        pos = s_len[r] + x - (s_end[r] - s_add[r]);
        const int pg = pos >> a.page_log2, fresh = pg - s_have[r];
        const int id = fresh >= 0 ? a.free_ring[ring_at(s_upto[r] - s_need[r] + fresh)]
                                  : a.tables[static_cast<int64_t>(r) * a.max_pages + pg];
        slot = (static_cast<int64_t>(id) << a.page_log2) + (pos & (P - 1));
      }
    }
    a.positions[x] = pos;
    a.slots[x] = slot;
  }
  // New page table entries (entries of refused requests lie past `taken`).
  for (int x = first; x < taken; x += stride) {
    const int r = first_above(s_upto, n, x);
    a.tables[static_cast<int64_t>(r) * a.max_pages + s_have[r] + x - (s_upto[r] - s_need[r])] = a.free_ring[ring_at(x)];
  }
  // Pages of the requests that have ended.
  for (int x = first; x < given_back; x += stride) {
    const int r = first_above(s_back, n, x);
    const int j = x - (s_back[r] - max(s_have[r] - a.prefix_pages, 0));
    a.free_ring[ring_at(count + x)] = a.tables[static_cast<int64_t>(r) * a.max_pages + a.prefix_pages + j];
  }
}

}  // namespace

hipError_t launch_kv_plan(const KvPlanArgs& a, hipStream_t st) {
  const int blocks = std::clamp((a.max_tokens + kPlanThreads - 1) / kPlanThreads, 1, 64);
  hipLaunchKernelGGL(kv_plan_kernel, dim3(blocks), dim3(kPlanThreads), 0, st, a);
  return hipGetLastError();
}

}  // namespace qm
