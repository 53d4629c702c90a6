// Eviction from a paged cache by accumulated attention weight: per sequence the forced tokens (sinks,
// recent ones) and the largest masses up to the budget, then a row gather into new pages.
//
// The choice is a radix selection on the 32-bit image of the mass (Eq. 14), most significant eight bits first:
// after four counting passes the threshold key and the number of tokens to take among the ones equal to it are known, and
// two ordered passes count and write the kept indices.  One work-group per sequence, bound by the latency of its passes over
// 4 bytes per token (eight loads in flight per thread); the gather that follows is bound by memory.
#include "up_attn.h"
#include "up_select.h"

namespace up {

namespace {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64, kEvictFly = 8;

// (a mass of -0 counts as 0)
__device__ __forceinline__ unsigned phi_of(float mass) { return phi(mass + 0.0f); }

__global__ __launch_bounds__(kEvictThreads) void k_evict_select(EvictArgs a) {
  __shared__ unsigned hist[kEvictWaves][256];
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
    for (int i0 = lo + tid; i0 < hi; i0 += kEvictFly * kEvictThreads) {
      float v[kEvictFly];
#pragma unroll
      for (int u = 0; u < kEvictFly; ++u) v[u] = mass[imin(i0 + u * kEvictThreads, hi - 1)];
#pragma unroll
      for (int u = 0; u < kEvictFly; ++u) {
        const unsigned key = phi_of(v[u]);
        if (i0 + u * kEvictThreads < hi && (key & mask) == prefix) atomicAdd(&hist[wave][(key >> shift) & 255u], 1u);
      }
    }
    __syncthreads();
    if (tid < 256) {
      unsigned sum = 0;
      for (int w = 0; w < kEvictWaves; ++w) sum += hist[w][tid];
      hist[0][tid] = sum;
    }
    __syncthreads();
    if (wave == 0) {
      // the digit at which the count from above reaches `left`: lane l holds digits 255 - 4l downwards
      unsigned n[4], mine = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        n[j] = hist[0][255 - 4 * lane - j];
        mine += n[j];
      }
      unsigned upto = mine;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned other = __shfl_up(upto, d);
        if (lane >= d) upto += other;
      }
      unsigned above = upto - mine;
      if (above < left && upto >= left) {      // (one lane: the counts add up to at least `left`)
        int j = 0;
        while (above + n[j] < left) above += n[j++];
        s_digit = (unsigned)(255 - 4 * lane - j);
        s_left = left - above;
      }
      if (left == 0 && lane == 0) {            // none is taken: no key may lie above the threshold
        s_digit = 255u;
        s_left = 0u;
      }
    }
    __syncthreads();
    prefix |= s_digit << shift;
    mask |= 255u << shift;
    left = s_left;
  }
  // prefix: key of the last token that stays; `left` of the tokens with this key stay, the lower indices.
  // Every wave takes a run of consecutive tokens, counts, and writes at its place.
  const int run = ((len + kEvictWaves - 1) / kEvictWaves + 63) / 64 * 64;
  const int w0 = wave * run, w1 = imin(len, w0 + run);
  constexpr int FLY = 4;
  int above = 0, equal = 0;
  for (int i0 = w0; i0 < w1; i0 += 64 * FLY) {
    float v[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) v[u] = mass[imin(i0 + u * 64 + lane, len - 1)];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const int i = i0 + u * 64 + lane;
      const unsigned key = phi_of(v[u]);
      const bool in = i < w1 && i >= lo && i < hi, forced = i < w1 && !in;
      above += __popcll(__ballot(forced || (in && key > prefix)));
      equal += __popcll(__ballot(in && key == prefix));
    }
  }
  if (lane == 0) { s_above[wave] = above; s_equal[wave] = equal; }
  __syncthreads();
  int out = 0, seen = 0;
  for (int w = 0; w < wave; ++w) { out += s_above[w]; seen += s_equal[w]; }
  out += imin(seen, (int)left);
  const unsigned long long below = (1ull << lane) - 1;
  for (int i0 = w0; i0 < w1; i0 += 64 * FLY) {
    float v[FLY];
#pragma unroll
    for (int u = 0; u < FLY; ++u) v[u] = mass[imin(i0 + u * 64 + lane, len - 1)];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const int i = i0 + u * 64 + lane;
      const unsigned key = phi_of(v[u]);
      const bool in = i < w1 && i >= lo && i < hi;
      const unsigned long long eq = __ballot(in && key == prefix);
      const bool keep = (i < w1 && !in) || (in && key > prefix) || (in && key == prefix && seen + __popcll(eq & below) < (int)left);
      const unsigned long long keeps = __ballot(keep);
      if (keep) {
        const int at = out + __popcll(keeps & below);
        kept[at] = i;
        mass_out[at] = v[u];
      }
      out += __popcll(keeps);
      seen += __popcll(eq);
    }
  }
}

// The kept rows of a sequence as 16-byte pieces in a row, four of them of both caches per thread in flight.
constexpr int kEvictPieces = 4;
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a) {
  const int r = blockIdx.y;
  const int kept = imin(imin(imax(a.kv_len[r], 0), a.max_len), a.budget);
  const unsigned pieces = (unsigned)(a.row_bytes / 16);
  const unsigned first = blockIdx.x * (256u * kEvictPieces) + threadIdx.x;
  long long src[kEvictPieces], dst[kEvictPieces];
  bool live[kEvictPieces];
#pragma unroll
  for (int u = 0; u < kEvictPieces; ++u) {
    unsigned j, piece, blk, at;
    divmod_by(first + u * 256u, pieces, a.piece_magic, j, piece);
    live[u] = j < (unsigned)kept;
    src[u] = dst[u] = 0;
    if (live[u]) {
      divmod_by((unsigned)a.kept_idx[(long long)r * a.mass_out_stride + j], (unsigned)a.kv_block, a.kv_magic, blk, at);
      src[u] = ((long long)a.block_table[(long long)r * a.table_stride + blk] * a.kv_block + at) * a.cache_stride + piece * 16;
      divmod_by(j, (unsigned)a.kv_block, a.kv_magic, blk, at);
      dst[u] = ((long long)a.new_table[(long long)r * a.new_table_stride + blk] * a.kv_block + at) * a.cache_stride + piece * 16;
    }
  }
  u32x4 k[kEvictPieces], v[kEvictPieces];
#pragma unroll
  for (int u = 0; u < kEvictPieces; ++u)
    if (live[u]) {
      k[u] = __builtin_nontemporal_load((const u32x4*)(a.k + src[u]));
      if (a.v != nullptr) v[u] = __builtin_nontemporal_load((const u32x4*)(a.v + src[u]));
    }
#pragma unroll
  for (int u = 0; u < kEvictPieces; ++u)
    if (live[u]) {
      __builtin_nontemporal_store(k[u], (u32x4*)(a.k + dst[u]));
      if (a.v != nullptr) __builtin_nontemporal_store(v[u], (u32x4*)(a.v + dst[u]));
    }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(k_evict_select, dim3(a.R), dim3(kEvictThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int most = a.budget < a.max_len ? a.budget : a.max_len;
  if (most > 0) {
    const long long pieces = (long long)most * (a.row_bytes / 16), each = 256 * kEvictPieces;
    hipLaunchKernelGGL(k_evict_move, dim3((unsigned)((pieces + each - 1) / each), a.R), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace up
