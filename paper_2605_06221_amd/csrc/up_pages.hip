// Pages for a step's new tokens: block table, offsets, positions and slots from the requests' lengths.
//
// Sequence r with len tokens in pages of B receives n more: it needs ceil((len + n) / B) - ceil(len / B) pages, the next ones from the
// end of the free list.  A prefix sum over the sequences says which; the first sequence that cannot be served ends the service (a rule
// that does not depend on the order in which work-groups run).  Bound by latency: one work-group adds up the sequences, 1024 at a
// time, and hands out the pages; the tokens' slots are looked up by as many lanes as there are tokens.
#include "up_layers.h"

namespace up {

constexpr int kPagesThreads = 1024, kPagesWaves = kPagesThreads / 64;

// inclusive sums of x over the work-group (every thread gets its own)
__device__ __forceinline__ long long pages_scan(long long x, long long* sm) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(x, d);
    if (lane >= d) x += o;
  }
  if (lane == 63) sm[wave] = x;
  __syncthreads();
  for (int w = 0; w < wave; ++w) x += sm[w];
  return x;
}

__global__ __launch_bounds__(kPagesThreads) void k_pages(PagesArgs a) {
  __shared__ long long sm[3][kPagesWaves];
  __shared__ long long ends[3];                 // sums of the round's served sequences
  __shared__ int first_bad;
  __shared__ int page_end[kPagesThreads], page_old[kPagesThreads];
  const int tid = threadIdx.x;
  const long long free_at_start = imax(0, a.num_free[0]);
  long long pages = 0, tokens = 0, keys = 0;      // of the rounds before
  int served = 0;
  bool going = true;
  if (tid == 0) { a.cu[0] = 0; a.cu_k[0] = 0; }
  for (int r0 = 0; r0 < a.R; r0 += kPagesThreads) {
    const int r = r0 + tid;
    long long len = 0, add = 0;
    if (r < a.R) {
      len = imax(0, a.kv_len[r]);
      add = imax(0, a.num_new[r]);
    }
    const long long old = (len + a.kv_block - 1) / a.kv_block, need = (len + add + a.kv_block - 1) / a.kv_block - old;
    if (tid == 0) { first_bad = going ? kPagesThreads : 0; ends[0] = ends[1] = 0; }
    const long long upto_pages = pages_scan(need, sm[0]), upto_tokens = pages_scan(add, sm[1]);
    const bool fits = pages + upto_pages <= free_at_start && tokens + upto_tokens <= a.capacity && old + need <= a.table_stride &&
                      len + add <= INT32_MAX;
    if (r < a.R && !fits) atomicMin(&first_bad, tid);
    __syncthreads();
    const int bad = first_bad, here = imin(bad, imin(kPagesThreads, a.R - r0));      // sequences served in this round
    if (tid == here - 1) { ends[0] = upto_pages; ends[1] = upto_tokens; }
    const bool mine = tid < here;
    const long long upto_keys = pages_scan(len + (mine ? add : 0), sm[2]);
    if (tid == kPagesThreads - 1) ends[2] = upto_keys;
    page_end[tid] = (int)upto_pages;      // (below 2^31 for the served ones, the only ones that are looked at)
    page_old[tid] = (int)old;
    __syncthreads();
    if (r < a.R) {
      a.new_len[r] = (int)(len + (mine ? add : 0));
      a.cu[r + 1] = (int)(tokens + (mine ? upto_tokens : ends[1]));
      const long long k = keys + upto_keys;
      a.cu_k[r + 1] = k > INT32_MAX ? INT32_MAX : (int)k;
    }
    const int handed = (int)ends[0];
    for (int e = tid; e < handed; e += kPagesThreads) {
      int lo = 0, hi = here - 1;      // the first sequence whose pages end behind e
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (page_end[mid] > e) hi = mid; else lo = mid + 1;
      }
      const int before = lo > 0 ? page_end[lo - 1] : 0;
      a.block_table[(long long)(r0 + lo) * a.table_stride + page_old[lo] + (e - before)] = a.free_pages[free_at_start - 1 - pages - e];
    }
    pages += ends[0];
    tokens += ends[1];
    keys += ends[2];
    served += here;
    going = going && here == imin(kPagesThreads, a.R - r0);
    __syncthreads();
  }
  if (tid == 0) {
    a.free_left[0] = (int)(free_at_start - pages);
    a.served[0] = served;
  }
}

// Positions and slots of the new tokens; what is left of the capacity is padding.
__global__ __launch_bounds__(256) void k_pages_slots(PagesArgs a) {
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  if (t >= a.capacity) return;
  int p = 0;
  int64_t slot = -1;
  if (a.R > 0 && t < (long long)a.cu[a.R]) {
    const int r = locate_token(a.cu, a.R, (int)t);
    p = a.new_len[r] - (a.cu[r + 1] - (int)t);
    slot = (int64_t)a.block_table[(long long)r * a.table_stride + p / a.kv_block] * a.kv_block + p % a.kv_block;
  }
  a.pos[t] = p;
  a.slots[t] = slot;
}

hipError_t launch_pages(const PagesArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_pages, dim3(1), dim3(kPagesThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.capacity == 0) return e;
  hipLaunchKernelGGL(k_pages_slots, dim3((unsigned)((a.capacity + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace up
