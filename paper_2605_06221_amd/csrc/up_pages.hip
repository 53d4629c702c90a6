// Pages for a step's new tokens: block table, offsets, positions and slots from the requests' lengths.
//
// Sequence r with len tokens in pages of B receives n more: it needs ceil((len + n) / B) - ceil(len / B) pages, the next ones from the
// end of the free list.  A prefix sum over the sequences says which; the first sequence that cannot be served ends the service (a rule
// that does not depend on the order in which work-groups run).  Bound by latency: one work-group adds up the sequences, 1024 or 4096 at a
// time, and hands out the pages; the tokens' slots are looked up by as many lanes as there are tokens.
// 64 sequences of one token: 7 us; 1200 sequences, 131300 tokens, 8400 pages: 20 us, 16 of them the one work-group's.
#include "up_attn.h"
#include "up_layers.h"

namespace up {

constexpr int kPagesThreads = 1024, kPagesWaves = kPagesThreads / 64;
constexpr int kPagesFew = 4096;      // tokens up to which one launch does both, of 1024 sequences at most
constexpr int kPagesSmall = 4096;    // sequences whose offsets are searched in LDS

// inclusive sums of x over the work-group (every thread gets its own), in two steps around a barrier
__device__ __forceinline__ long long pages_scan_wave(long long x, long long* sm) {
  const int lane = threadIdx.x & 63;
  for (int d = 1; d < 64; d <<= 1) {
    const long long o = __shfl_up(x, d);
    if (lane >= d) x += o;
  }
  if (lane == 63) sm[threadIdx.x >> 6] = x;
  return x;
}
__device__ __forceinline__ long long pages_scan_rest(long long x, const long long* sm) {
  const int wave = threadIdx.x >> 6;
#pragma unroll
  for (int w = 0; w < kPagesWaves; ++w) x += w < wave ? sm[w] : 0;
  return x;
}

// pages that n tokens take
__device__ __forceinline__ int pages_of(const PagesArgs& a, int n) {
  unsigned whole, rest;
  divmod_by((unsigned)n, (unsigned)a.kv_block, a.kv_magic, whole, rest);
  return (int)whole + (rest != 0);
}

// The position of the token at place p of sequence r's cache: the tokens that the cache does not hold stand before it.
__device__ __forceinline__ int pages_position(const PagesArgs& a, int r, int p) {
  if (a.dropped == nullptr) return p;
  const long long at = (long long)p + imax(0, a.dropped[r]);
  return at > INT32_MAX ? INT32_MAX : (int)at;
}

// the first of n ends that lies behind x
__device__ __forceinline__ int first_past(const int* end, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (end[mid] > x) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// EACH: sequences of a thread in a round (a round costs some 5 us, one with four sequences a thread 2 us more)
template <int EACH>
__global__ __launch_bounds__(kPagesThreads) void k_pages(PagesArgs a) {
  constexpr int ROUND = kPagesThreads * EACH;
  __shared__ long long sm[3][kPagesWaves];
  __shared__ long long ends[2];                 // pages and tokens of the round's served sequences
  __shared__ int first_bad;
  __shared__ int page_end[ROUND], page_old[ROUND], token_end[ROUND], new_len[ROUND];
  const int tid = threadIdx.x;
  const long long free_at_start = imax(0, a.num_free[0]);
  long long pages = 0, tokens = 0, keys = 0;      // of the rounds before
  int served = 0;
  bool going = true;
  if (tid == 0) { a.cu[0] = 0; a.cu_k[0] = 0; }
  for (int r0 = 0; r0 < a.R; r0 += ROUND) {
    const int here0 = imin(ROUND, a.R - r0), first = tid * EACH;      // (the thread's sequences: first .. of the round)
    int len[EACH], old[EACH], need[EACH];
    long long add[EACH], my_pages = 0, my_tokens = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const bool there = first + i < here0;
      len[i] = there ? imax(0, a.kv_len[r0 + first + i]) : 0;
      add[i] = there ? imax(0, a.num_new[r0 + first + i]) : 0;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      old[i] = pages_of(a, len[i]);
      need[i] = len[i] + add[i] <= INT32_MAX ? pages_of(a, (int)(len[i] + add[i])) - old[i] : 0;      // (else it is not served, whatever it needs)
      my_pages += need[i];
      my_tokens += add[i];
    }
    if (tid == 0) { first_bad = going ? here0 : 0; ends[0] = ends[1] = 0; }
    long long upto_pages = pages_scan_wave(my_pages, sm[0]), upto_tokens = pages_scan_wave(my_tokens, sm[1]);
    __syncthreads();
    upto_pages = pages_scan_rest(upto_pages, sm[0]) - my_pages;
    upto_tokens = pages_scan_rest(upto_tokens, sm[1]) - my_tokens;
    int bad = here0;
    long long p = upto_pages, t = upto_tokens;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      p += need[i];
      t += add[i];
      const bool fits = pages + p <= free_at_start && tokens + t <= a.capacity && (long long)old[i] + need[i] <= a.table_stride &&
                        len[i] + add[i] <= INT32_MAX;
      if (!fits) bad = imin(bad, first + i);
    }
    if (bad < here0) atomicMin(&first_bad, bad);
    __syncthreads();
    const int here = first_bad;      // sequences served in this round
    long long my_keys = 0;
    p = upto_pages;
    t = upto_tokens;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      p += need[i];
      t += add[i];
      if (first + i == here - 1) { ends[0] = p; ends[1] = t; }
      page_end[first + i] = (int)p;      // (below 2^31 for the served ones, the only ones that are looked at)
      page_old[first + i] = old[i];
      token_end[first + i] = (int)t;
      new_len[first + i] = (int)(len[i] + (first + i < here ? add[i] : 0));
      my_keys += new_len[first + i];
    }
    long long upto_keys = pages_scan_wave(my_keys, sm[2]);
    __syncthreads();
    upto_keys = keys + pages_scan_rest(upto_keys, sm[2]) - my_keys;
    long long all_keys = 0;
#pragma unroll
    for (int w = 0; w < kPagesWaves; ++w) all_keys += sm[2][w];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int s = first + i;
      if (s >= here0) break;
      upto_keys += new_len[s];
      a.new_len[r0 + s] = new_len[s];
      a.cu[r0 + s + 1] = (int)(tokens + (s < here ? token_end[s] : ends[1]));
      a.cu_k[r0 + s + 1] = upto_keys > INT32_MAX ? INT32_MAX : (int)upto_keys;
    }
    const int handed = (int)ends[0];
    // Eight pages a thread at a time, their loads under way together; neighbouring lanes take neighbouring pages (a thread for a row of them:
    // 64 lines a store instead of some ten, 17 -> 28 us for 8400 pages).
    for (int e0 = tid; e0 < handed; e0 += 8 * kPagesThreads) {
      int page[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = e0 + i * kPagesThreads;
        page[i] = e < handed ? a.free_pages[free_at_start - 1 - pages - e] : 0;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int e = e0 + i * kPagesThreads;
        if (e >= handed) break;
        const int s = first_past(page_end, here, e);
        a.block_table[(long long)(r0 + s) * a.table_stride + page_old[s] + (e - (s > 0 ? page_end[s - 1] : 0))] = page[i];
      }
    }
    if (a.one_launch) {      // (one round, so the sums start at 0)
      for (int t = tid; t < (int)a.capacity; t += kPagesThreads) {
        int p = 0;
        int64_t slot = -1;
        if (t < (int)ends[1]) {
          const int s = first_past(token_end, here, t);
          const int add = token_end[s] - (s > 0 ? token_end[s - 1] : 0);
          p = new_len[s] - (token_end[s] - t);
          unsigned j, at;
          divmod_by((unsigned)p, (unsigned)a.kv_block, a.kv_magic, j, at);
          const unsigned had = (unsigned)pages_of(a, new_len[s] - add);
          const int id = j < had ? a.block_table[(long long)s * a.table_stride + j]
                                 : a.free_pages[free_at_start - 1 - (s > 0 ? page_end[s - 1] : 0) - (int)(j - had)];
          slot = (int64_t)id * a.kv_block + at;
          p = pages_position(a, s, p);
        }
        a.pos[t] = p;
        a.slots[t] = slot;
      }
    }
    pages += ends[0];
    tokens += ends[1];
    keys += all_keys;
    served += here;
    going = going && here == here0;
    __syncthreads();
  }
  if (tid == 0) {
    a.free_left[0] = (int)(free_at_start - pages);
    a.served[0] = served;
  }
}

// Positions and slots of the new tokens; what is left of the capacity is padding.  SMALL: the offsets fit the LDS, and a token's search
// for its sequence does not go through memory step by step.
template <bool SMALL>
__global__ __launch_bounds__(256) void k_pages_slots(PagesArgs a) {
  __shared__ int ends[SMALL ? kPagesSmall : 1];
  const long long t = (long long)blockIdx.x * 256 + threadIdx.x;
  if (SMALL) {
    for (int r = threadIdx.x; r < a.R; r += 256) ends[r] = a.cu[r + 1];
    __syncthreads();
  }
  if (t >= a.capacity) return;
  int p = 0;
  int64_t slot = -1;
  if (a.R > 0 && t < (long long)(SMALL ? ends[a.R - 1] : a.cu[a.R])) {
    const int r = SMALL ? first_past(ends, a.R, (int)t) : locate_token(a.cu, a.R, (int)t);
    p = a.new_len[r] - ((SMALL ? ends[r] : a.cu[r + 1]) - (int)t);
    unsigned j, at;
    divmod_by((unsigned)p, (unsigned)a.kv_block, a.kv_magic, j, at);
    slot = (int64_t)a.block_table[(long long)r * a.table_stride + j] * a.kv_block + at;
    p = pages_position(a, r, p);
  }
  a.pos[t] = p;
  a.slots[t] = slot;
}

hipError_t launch_pages(const PagesArgs& args, hipStream_t s) {
  // few tokens are looked up by the work-group that handed out their pages, in the same launch
  PagesArgs a = args;
  a.one_launch = a.R > 0 && a.R <= kPagesThreads && a.capacity <= kPagesFew;
  if (a.R <= kPagesThreads) hipLaunchKernelGGL(k_pages<1>, dim3(1), dim3(kPagesThreads), 0, s, a);
  else hipLaunchKernelGGL(k_pages<4>, dim3(1), dim3(kPagesThreads), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.capacity == 0 || a.one_launch) return e;
  const dim3 grid((unsigned)((a.capacity + 255) / 256));
  if (a.R <= kPagesSmall) hipLaunchKernelGGL(k_pages_slots<true>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_pages_slots<false>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace up
