// Eviction from a paged cache by accumulated attention weight: per sequence the forced tokens (sinks,
// recent ones) and the largest masses up to the budget, then a row gather into new pages.
//
// The choice is a radix selection on the 32-bit image of the mass (Eq. 14), most significant eight bits first:
// after four counting passes the threshold key and the number of tokens to take among the ones equal to it are known, and one
// ordered pass writes the kept indices.  Bound by latency: a few passes over 4 bytes per token by one work-group.
#include "up_attn.h"
#include "up_copy.h"
#include "up_select.h"

namespace up {

namespace {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;

// (a mass of -0 counts as 0)
__device__ __forceinline__ unsigned phi_of(float mass) { return phi(mass + 0.0f); }

__global__ __launch_bounds__(kEvictThreads) void k_evict_select(EvictArgs a) {
  __shared__ unsigned hist[kEvictWaves][256];
  __shared__ unsigned total[256];
  __shared__ unsigned s_digit, s_left;
  __shared__ int s_above[kEvictWaves], s_equal[kEvictWaves];
  const int r = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  const float* mass = a.mass + (long long)r * a.mass_stride;
  int32_t* kept = a.kept_idx + (long long)r * a.mass_out_stride;
  float* mass_out = a.mass_out + (long long)r * a.mass_out_stride;
  if (tid == 0) a.new_len[r] = imin(len, a.budget);
  if (len <= a.budget) {
    for (int i = tid; i < len; i += kEvictThreads) {
      kept[i] = i;
      mass_out[i] = mass[i];
    }
    return;
  }
  const int lo = a.n_sink, hi = len - a.n_recent;      // the tokens that compete (lo < hi: the budget is below len)
  const int take = a.budget - a.n_sink - a.n_recent;   // how many of them stay
  unsigned prefix = 0, mask = 0, left = (unsigned)take;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < kEvictWaves * 256; i += kEvictThreads) (&hist[0][0])[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kEvictThreads) {
      const unsigned key = phi_of(mass[i]);
      if ((key & mask) == prefix) atomicAdd(&hist[wave][(key >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (tid < 256) {
      unsigned sum = 0;
      for (int w = 0; w < kEvictWaves; ++w) sum += hist[w][tid];
      total[tid] = sum;
    }
    __syncthreads();
    if (tid == 0) {
      // the digit at which the count from above reaches `left`
      unsigned n = left;
      int d = 255;
      while (d > 0 && total[d] < n) { n -= total[d]; --d; }
      s_digit = (unsigned)d;
      s_left = n;
    }
    __syncthreads();
    prefix |= s_digit << shift;
    mask |= 255u << shift;
    left = s_left;
  }
  // prefix: key of the last token that stays; `left` of the tokens with this key stay, the lower indices.  (take == 0:
  // left stays 0 and no key lies above the all-ones prefix that the passes then end with.)
  // Every wave takes a run of consecutive tokens, counts, and writes at its place.
  const int run = ((len + kEvictWaves - 1) / kEvictWaves + 63) / 64 * 64;
  const int w0 = wave * run, w1 = imin(len, w0 + run);
  int above = 0, equal = 0;
  for (int i0 = w0; i0 < w1; i0 += 64) {
    const int i = i0 + lane;
    const unsigned key = i >= lo && i < hi ? phi_of(mass[i]) : 0u;
    const bool in = i < w1 && i >= lo && i < hi;
    const bool forced = i < w1 && !in;
    above += __popcll(__ballot(forced || (in && key > prefix)));
    equal += __popcll(__ballot(in && key == prefix));
  }
  if (lane == 0) { s_above[wave] = above; s_equal[wave] = equal; }
  __syncthreads();
  int out = 0, seen = 0;
  for (int w = 0; w < wave; ++w) { out += s_above[w]; seen += s_equal[w]; }
  out += imin(seen, (int)left);
  const unsigned long long below = (1ull << lane) - 1;
  for (int i0 = w0; i0 < w1; i0 += 64) {
    const int i = i0 + lane;
    const bool in = i < w1 && i >= lo && i < hi;
    const float v = i < w1 ? mass[i] : 0.0f;
    const unsigned key = phi_of(v);
    const unsigned long long eq = __ballot(in && key == prefix);
    const bool keep = (i < w1 && !in) || (in && key > prefix) ||
                      (in && key == prefix && seen + __popcll(eq & below) < (int)left);
    const unsigned long long keeps = __ballot(keep);
    if (keep) {
      const int at = out + __popcll(keeps & below);
      kept[at] = i;
      mass_out[at] = v;
    }
    out += __popcll(keeps);
    seen += __popcll(eq);
  }
}

// One wave per kept token: its rows of both caches into the new page.
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int r = blockIdx.y, j = blockIdx.x * 4 + wave;
  if (j >= imin(imin(imax(a.kv_len[r], 0), a.max_len), a.budget)) return;
  unsigned blk, at;
  divmod_by((unsigned)a.kept_idx[(long long)r * a.mass_out_stride + j], (unsigned)a.kv_block, a.kv_magic, blk, at);
  const long long src = ((long long)a.block_table[(long long)r * a.table_stride + blk] * a.kv_block + at) * a.cache_stride;
  divmod_by((unsigned)j, (unsigned)a.kv_block, a.kv_magic, blk, at);
  const long long dst = ((long long)a.new_table[(long long)r * a.new_table_stride + blk] * a.kv_block + at) * a.cache_stride;
  copy_row_wave(a.k + src, a.k + dst, a.row_bytes, lane);
  if (a.v != nullptr) copy_row_wave(a.v + src, a.v + dst, a.row_bytes, lane);
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_evict_select, dim3(a.R), dim3(kEvictThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int most = a.budget < a.max_len ? a.budget : a.max_len;
  if (most > 0) {
    hipLaunchKernelGGL(k_evict_move, dim3((most + 3) / 4, a.R), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace up
