// Eviction from a paged cache by accumulated attention weight: per sequence the forced tokens (sinks,
// recent ones) and the largest masses up to the budget, then a row gather into new pages.
//
// The choice is a radix selection on the 32-bit image of the mass (Eq. 14) by a histogram of its first twelve bits and two of ten.
// One work-group per sequence puts the few tokens of the threshold's first digit aside in LDS, as their other twenty bits and the wave
// they came from, and counts the other two digits and every wave's share there.  Long sequences (kEvictLong) are counted by
// many work-groups, one launch per digit.  The gather that follows is bound by memory.
#include "up_attn.h"
#include "up_select.h"

namespace up {

namespace {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64, kEvictFly = 8;
// A longest sequence (by max_kv_len: the lengths are on the device) from which on many work-groups choose, where the budget leaves them room
// to count in a row of mass_out, kSpreadCounts + 2 words a work-group, 6152 + 2 * max_kv_len / 4096; below that one work-group has to
// (131072 tokens: 57 us to 16384, 111 to 4096, 101 to 1024).  Their six launches cost what one
// work-group takes for 24576 tokens (with the move and reading back 8000 rows: 16384 tokens 37 against 43 us, 24576 43.4 and 43.6, 32768
// 49.5 against 43.7, 131072 136 against 59, 200000 171 against 45).
constexpr int kEvictLong = 24576;
constexpr int kEvictRest = 24576;   // tokens that share the first digit and fit LDS; more of them are counted from memory

// (a mass of -0 counts as 0)
__device__ __forceinline__ unsigned phi_of(float mass) { return phi(mass + 0.0f); }

// one more of digit `d`: a wave of equal digits (tokens that no one looked at yet share their mass) adds once
__device__ __forceinline__ void count_digit(unsigned* hist, bool in, unsigned d) {
  const unsigned long long who = __ballot(in);
  if (who == 0) return;
  const unsigned one = (unsigned)__builtin_amdgcn_readlane((int)d, __builtin_ctzll(who));
  if (__ballot(in && d == one) == who) {
    if ((int)(threadIdx.x & 63) == __builtin_ctzll(who)) atomicAdd(&hist[one], (unsigned)__popcll(who));
  } else if (in) {
    atomicAdd(&hist[d], 1u);
  }
}

// The digit at which the count from the highest one down reaches `left` (1 .. all): f.digit, how many are left to take with
// that digit (f.left), and how many tokens have it (f.count).  THREADS * PER digits.
struct EvictFind {
  unsigned total[kEvictWaves];
  unsigned digit, left, count;
};
template <int THREADS, int PER>
__device__ __forceinline__ void find_digit(EvictFind& f, const unsigned* hist, unsigned left) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  unsigned n[PER], mine = 0;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    n[j] = hist[PER * THREADS - 1 - PER * tid - j];
    mine += n[j];
  }
  unsigned upto = mine;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const unsigned other = __shfl_up(upto, d);
    if (lane >= d) upto += other;
  }
  if (lane == 63) f.total[wave] = upto;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) upto += w < wave ? f.total[w] : 0u;
  unsigned above = upto - mine;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if (above < left && above + n[j] >= left) {      // one thread, one j
      f.digit = (unsigned)(PER * THREADS - 1 - PER * tid - j);
      f.left = left - above;
      f.count = n[j];
    }
    above += n[j];
  }
  __syncthreads();
}

struct EvictLds {
  unsigned hist[4096 + 2 * 1024];      // of the three digits
  unsigned rest[kEvictRest];
  EvictFind find;
  unsigned n_rest, lowest, highest;
  unsigned above[kEvictWaves], equal[kEvictWaves];
};

// One work-group, bound by the issue of its instructions: of the 8.9 us for 4096 tokens, 1.2 go to the first histogram, 2.7 to putting the tokens of the
// threshold's digit aside, 2 to the other digits, 2.2 to writing.  HELD: a wave's run of tokens is one group of kEvictFly * 64, read once.
template <bool HELD>
__device__ __forceinline__ void evict_select(const EvictArgs& a, EvictLds& s, const float* mass, int len, int run, int32_t* kept, float* mass_out) {
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int lo = a.n_sink, hi = len - a.n_recent;      // the tokens that compete (lo < hi: the budget is below len)
  unsigned left = (unsigned)(a.budget - a.n_sink - a.n_recent);   // how many of them stay
  const int w0 = imin(wave * run, len), w1 = imin(len, w0 + run);
  const int c0 = imax(w0, lo), competing = imax(imin(w1, hi) - c0, 0);
  float held[kEvictFly];
  auto load = [&](int g0, float* v) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kEvictFly; ++u) v[u] = mass[imin(g0 + u * 64 + lane, len - 1)];
  };
  auto groups = [&](auto f) __attribute__((always_inline)) {
    if constexpr (HELD) {
      if (w0 < w1) f(w0, held);
    } else {
      for (int g0 = w0; g0 < w1; g0 += kEvictFly * 64) {
        float v[kEvictFly];
        load(g0, v);
        f(g0, v);
      }
    }
  };
  auto competes = [&](int g0, int u) __attribute__((always_inline)) { return (unsigned)(g0 + u * 64 + lane - c0) < (unsigned)competing; };
  if constexpr (HELD) load(w0, held);
  unsigned *first = s.hist, *second = s.hist + 4096, *third = s.hist + 4096 + 1024;
  for (int i = tid; i < 4096 + 2 * 1024; i += kEvictThreads) s.hist[i] = 0;
  if (tid < kEvictWaves) s.above[tid] = s.equal[tid] = 0;
  if (tid == 0) {
    s.n_rest = s.highest = 0;
    s.lowest = ~0u;
  }
  __syncthreads();

  unsigned bar = ~0u;      // the key of the last token that stays; `left` of the tokens with this key stay, the lower indices
  if (left != 0) {
    groups([&](int g0, const float* v) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < kEvictFly; ++u) count_digit(first, competes(g0, u), phi_of(v[u]) >> 20);
    });
    __syncthreads();
    find_digit<kEvictThreads, 4>(s.find, first, left);
    const unsigned top = s.find.digit, n_rest = s.find.count;
    left = s.find.left;
    const bool fits = n_rest <= (unsigned)kEvictRest;
    bool done = false;
    if (fits) {
      unsigned above = 0;
      groups([&](int g0, const float* v) __attribute__((always_inline)) {
        unsigned n = 0;
        unsigned long long same[kEvictFly];
#pragma unroll
        for (int u = 0; u < kEvictFly; ++u) {
          const unsigned d = phi_of(v[u]) >> 20;
          const bool in = competes(g0, u);
          above += __popcll(__ballot(in && d > top));
          same[u] = __ballot(in && d == top);
          n += __popcll(same[u]);
        }
        if (n == 0) return;
        unsigned at = 0;
        if (lane == 0) at = atomicAdd(&s.n_rest, n);
        at = (unsigned)__builtin_amdgcn_readfirstlane((int)at);
#pragma unroll
        for (int u = 0; u < kEvictFly; ++u) {
          if ((same[u] >> lane) & 1) s.rest[at + __popcll(same[u] & ((1ull << lane) - 1))] = (phi_of(v[u]) & 0xfffffu) | ((unsigned)wave << 20);
          at += __popcll(same[u]);
        }
      });
      if (lane == 0) s.above[wave] = above;
      __syncthreads();
      for (unsigned i = tid; i < n_rest; i += kEvictThreads) count_digit(second, true, (s.rest[i] >> 10) & 1023u);
    } else {
      // more than fit are most often all one mass (nothing, of tokens that no row looked at): then it is the bar
      unsigned above = 0, equal = 0, lowest = ~0u, highest = 0;
      groups([&](int g0, const float* v) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < kEvictFly; ++u) {
          const unsigned key = phi_of(v[u]);
          const bool in = competes(g0, u), same = in && (key >> 20) == top;
          above += __popcll(__ballot(in && (key >> 20) > top));
          equal += __popcll(__ballot(same));
          lowest = same && key < lowest ? key : lowest;
          highest = same && key > highest ? key : highest;
        }
      });
      atomicMin(&s.lowest, lowest);
      atomicMax(&s.highest, highest);
      if (lane == 0) { s.above[wave] = above; s.equal[wave] = equal; }
      __syncthreads();
      done = s.lowest == s.highest;
      if (done) {
        bar = s.lowest;
      } else {
        groups([&](int g0, const float* v) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < kEvictFly; ++u) {
            const unsigned key = phi_of(v[u]);
            count_digit(second, competes(g0, u) && (key >> 20) == top, (key >> 10) & 1023u);
          }
        });
      }
    }
    if (!done) {
      __syncthreads();
      find_digit<kEvictThreads, 1>(s.find, second, left);
      const unsigned two = (top << 10) | s.find.digit;
      left = s.find.left;
      if (fits) {
        for (unsigned i = tid; i < n_rest; i += kEvictThreads) {
          const unsigned e = s.rest[i];
          count_digit(third, ((e >> 10) & 1023u) == (two & 1023u), e & 1023u);
        }
      } else {
        groups([&](int g0, const float* v) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < kEvictFly; ++u) {
            const unsigned key = phi_of(v[u]);
            count_digit(third, competes(g0, u) && (key >> 10) == two, key & 1023u);
          }
        });
      }
      __syncthreads();
      find_digit<kEvictThreads, 1>(s.find, third, left);
      bar = (two << 10) | s.find.digit;
      left = s.find.left;
      if (fits) {
        for (unsigned i = tid; i < n_rest; i += kEvictThreads) {
          const unsigned e = s.rest[i];
          count_digit(s.above, (e & 0xfffffu) > (bar & 0xfffffu), e >> 20);
          count_digit(s.equal, (e & 0xfffffu) == (bar & 0xfffffu), e >> 20);
        }
      } else {
        unsigned above = 0, equal = 0;
        groups([&](int g0, const float* v) __attribute__((always_inline)) {
#pragma unroll
          for (int u = 0; u < kEvictFly; ++u) {
            const unsigned key = phi_of(v[u]);
            above += __popcll(__ballot(competes(g0, u) && key > bar));
            equal += __popcll(__ballot(competes(g0, u) && key == bar));
          }
        });
        if (lane == 0) { s.above[wave] = above; s.equal[wave] = equal; }
      }
    }
    __syncthreads();
  }
  // a wave writes behind what the waves before it keep: their forced tokens, the ones above the bar, and their share of the equal ones
  const int before = imin(w0, lo) + imax(w0 - hi, 0);
  unsigned above = 0, seen = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    above += w < wave ? s.above[w] : 0u;
    seen += w < wave ? s.equal[w] : 0u;
  }
  int out = before + (int)above + imin((int)seen, (int)left);
  const unsigned long long below = (1ull << lane) - 1;
  groups([&](int g0, const float* v) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kEvictFly; ++u) {
      const int i = g0 + u * 64 + lane;
      const unsigned key = phi_of(v[u]);
      const bool in = competes(g0, u);
      const unsigned long long eq = __ballot(in && key == bar);
      const bool keep = (i < w1 && !in) || (in && key > bar) || (in && key == bar && seen + __popcll(eq & below) < left);
      const unsigned long long keeps = __ballot(keep);
      if (keep) {
        const int at = out + __popcll(keeps & below);
        kept[at] = i;
        mass_out[at] = v[u];
      }
      out += __popcll(keeps);
      seen += __popcll(eq);
    }
  });
}

__global__ __launch_bounds__(kEvictThreads) void k_evict_select(EvictArgs a) {
  __shared__ EvictLds s;
  const int r = blockIdx.x, tid = threadIdx.x;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  const float* mass = a.mass + (long long)r * a.mass_stride;
  int32_t* kept = a.kept_idx + (long long)r * a.mass_out_stride;
  float* mass_out = a.mass_out + (long long)r * a.mass_out_stride;
  if (len <= a.budget) {
    for (int i = tid; i < len; i += kEvictThreads) {
      kept[i] = i;
      mass_out[i] = mass[i];
    }
    return;
  }
  // every wave takes a run of consecutive tokens
  const int run = ((len + kEvictWaves - 1) / kEvictWaves + 63) / 64 * 64;
  if (run <= kEvictFly * 64)
    evict_select<true>(a, s, mass, len, run, kept, mass_out);
  else
    evict_select<false>(a, s, mass, len, run, kept, mass_out);
}

// Long sequences, WHAT after WHAT: the histograms of the three digits, every work-group's count of tokens above and at the bar, and the
// kept indices.  What passes from launch to launch lies in the sequence's row of mass_out, which the move fills at last: the histograms, the digits found
// so far with what is left to take (one pair per digit), and a pair of counts per work-group.
constexpr int kSpreadThreads = 256, kSpreadWaves = kSpreadThreads / 64, kSpreadEach = 16, kSpreadTokens = kSpreadThreads * kSpreadEach;
constexpr int kSpreadFound = 4096 + 2 * 1024, kSpreadCounts = kSpreadFound + 8;
enum { kClear, kFirst, kSecond, kThird, kCount, kWrite };

template <int WHAT>
__global__ __launch_bounds__(kSpreadThreads) void k_evict_spread(EvictArgs a) {
  __shared__ unsigned hist[WHAT == kFirst ? 4096 : 1024];
  __shared__ EvictFind find;
  __shared__ unsigned s_above[kSpreadWaves], s_equal[kSpreadWaves], s_before[2];
  const int r = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  const float* mass = a.mass + (long long)r * a.mass_stride;
  int32_t* kept = a.kept_idx + (long long)r * a.mass_out_stride;
  float* mass_out = a.mass_out + (long long)r * a.mass_out_stride;
  unsigned* scratch = (unsigned*)mass_out;
  const int from = (int)blockIdx.x * kSpreadTokens;
  if constexpr (WHAT == kClear) {
    if (len > a.budget)
      for (int i = (int)blockIdx.x * kSpreadThreads + tid; i < kSpreadFound; i += (int)gridDim.x * kSpreadThreads) scratch[i] = 0;
    return;
  }
  if (from >= len) return;
  if (len <= a.budget) {
    if (WHAT == kWrite) {
      for (int i = from + tid; i < imin(len, from + kSpreadTokens); i += kSpreadThreads) kept[i] = i;
    }
    return;
  }
  const int lo = a.n_sink, hi = len - a.n_recent;
  unsigned left = (unsigned)(a.budget - a.n_sink - a.n_recent);
  const int w0 = imin(from + wave * (kSpreadTokens / kSpreadWaves), len), w1 = imin(len, w0 + kSpreadTokens / kSpreadWaves);
  const int c0 = imax(w0, lo), competing = imax(imin(w1, hi) - c0, 0);
  float v[kSpreadEach];
#pragma unroll
  for (int u = 0; u < kSpreadEach; ++u) v[u] = mass[imin(w0 + u * 64 + lane, len - 1)];
  auto competes = [&](int u) __attribute__((always_inline)) { return (unsigned)(w0 + u * 64 + lane - c0) < (unsigned)competing; };

  if constexpr (WHAT <= kThird) {
    for (int i = tid; i < (WHAT == kFirst ? 4096 : 1024); i += kSpreadThreads) hist[i] = 0;
  }
  // the digits found before, and the one that the histogram of the launch before gives
  unsigned bar = 0;
  if constexpr (WHAT > kSecond && WHAT <= kCount) {
    bar = scratch[kSpreadFound + 2 * (WHAT - kThird)];
    left = scratch[kSpreadFound + 2 * (WHAT - kThird) + 1];
  }
  if constexpr (WHAT >= kSecond && WHAT <= kCount) {
    if constexpr (WHAT == kSecond) find_digit<kSpreadThreads, 16>(find, scratch, left);
    else find_digit<kSpreadThreads, 4>(find, scratch + 4096 + (WHAT - kThird) * 1024, left);
    bar = (bar << 10) | find.digit;
    left = find.left;
    if (from == 0 && tid == 0) {
      scratch[kSpreadFound + 2 * (WHAT - kSecond)] = bar;
      scratch[kSpreadFound + 2 * (WHAT - kSecond) + 1] = left;
    }
  } else if constexpr (WHAT == kWrite) {
    if (left == 0) {
      bar = ~0u;
    } else {
      bar = scratch[kSpreadFound + 4];
      left = scratch[kSpreadFound + 5];
    }
  }
  if constexpr (WHAT <= kThird) {
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kSpreadEach; ++u) {
      const unsigned key = phi_of(v[u]);
      if (WHAT == kFirst) count_digit(hist, competes(u), key >> 20);
      if (WHAT == kSecond) count_digit(hist, competes(u) && (key >> 20) == bar, (key >> 10) & 1023u);
      if (WHAT == kThird) count_digit(hist, competes(u) && (key >> 10) == bar, key & 1023u);
    }
    __syncthreads();
    unsigned* sum = scratch + (WHAT == kFirst ? 0 : 4096 + (WHAT - kSecond) * 1024);
    for (int i = tid; i < (WHAT == kFirst ? 4096 : 1024); i += kSpreadThreads)
      if (hist[i] != 0) atomicAdd(&sum[i], hist[i]);      // (whole numbers: any order gives the same)
    return;
  }
  unsigned above = 0, equal = 0;
#pragma unroll
  for (int u = 0; u < kSpreadEach; ++u) {
    const unsigned key = phi_of(v[u]);
    above += __popcll(__ballot(competes(u) && key > bar));
    equal += __popcll(__ballot(competes(u) && key == bar));
  }
  if (lane == 0) { s_above[wave] = above; s_equal[wave] = equal; }
  if constexpr (WHAT == kCount) {
    __syncthreads();
    if (tid == 0) {
      above = equal = 0;
      for (int w = 0; w < kSpreadWaves; ++w) { above += s_above[w]; equal += s_equal[w]; }
      scratch[kSpreadCounts + 2 * blockIdx.x] = above;
      scratch[kSpreadCounts + 2 * blockIdx.x + 1] = equal;
    }
    return;
  }
  // (kWrite) behind what the tokens before the wave's keep: the forced ones, the ones above the bar, their share of the equal ones
  if (tid < 2) s_before[tid] = 0;
  __syncthreads();
  if (left != 0) {
    unsigned n = 0;
    for (int i = tid; i < 2 * (int)blockIdx.x; i += kSpreadThreads) n += scratch[kSpreadCounts + i];
    if (n != 0) atomicAdd(&s_before[tid & 1], n);
  }
  __syncthreads();
  above = s_before[0];
  unsigned seen = s_before[1];
  for (int w = 0; w < wave; ++w) { above += s_above[w]; seen += s_equal[w]; }
  int out = imin(w0, lo) + imax(w0 - hi, 0) + (int)above + imin((int)seen, (int)left);
  const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
  for (int u = 0; u < kSpreadEach; ++u) {
    const int i = w0 + u * 64 + lane;
    const unsigned key = phi_of(v[u]);
    const bool in = competes(u);
    const unsigned long long eq = __ballot(in && key == bar);
    const bool keep = (i < w1 && !in) || (in && key > bar) || (in && key == bar && seen + __popcll(eq & below) < left);
    const unsigned long long keeps = __ballot(keep);
    if (keep) kept[out + __popcll(keeps & below)] = i;
    out += __popcll(keeps);
    seen += __popcll(eq);
  }
}

// The kept rows of a sequence as 16-byte pieces in a row, four of them of both caches per thread in flight, and how many rows they are.
// MASS: the kept masses too.
constexpr int kEvictPieces = 4;
template <bool MASS>
__global__ __launch_bounds__(256) void k_evict_move(EvictArgs a) {
  const int r = blockIdx.y;
  const int kept = imin(imin(imax(a.kv_len[r], 0), a.max_len), a.budget);
  // (new_len may be kv_len: of the length before and the one that is kept the same number follows, so any order will do)
  if (blockIdx.x == 0 && threadIdx.x == 0) a.new_len[r] = kept;
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
      const int i = a.kept_idx[(long long)r * a.mass_out_stride + j];
      if (MASS && piece == 0) a.mass_out[(long long)r * a.mass_out_stride + j] = a.mass[(long long)r * a.mass_stride + i];
      divmod_by((unsigned)i, (unsigned)a.kv_block, a.kv_magic, blk, at);
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
  const unsigned groups = (unsigned)((a.max_len + (long long)kSpreadTokens - 1) / kSpreadTokens);
  const bool spread = a.max_len >= kEvictLong && a.budget >= kSpreadCounts + 2ll * groups;
  if (spread) {
    const dim3 grid(groups, a.R), threads(kSpreadThreads);
    if (a.budget > a.n_sink + a.n_recent) {
      hipLaunchKernelGGL(k_evict_spread<kClear>, dim3(4, a.R), threads, 0, s, a);
      hipLaunchKernelGGL(k_evict_spread<kFirst>, grid, threads, 0, s, a);
      hipLaunchKernelGGL(k_evict_spread<kSecond>, grid, threads, 0, s, a);
      hipLaunchKernelGGL(k_evict_spread<kThird>, grid, threads, 0, s, a);
      hipLaunchKernelGGL(k_evict_spread<kCount>, grid, threads, 0, s, a);
    }
    hipLaunchKernelGGL(k_evict_spread<kWrite>, grid, threads, 0, s, a);
  } else {
    hipLaunchKernelGGL(k_evict_select, dim3(a.R), dim3(kEvictThreads), 0, s, a);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // (one work-group at least: it writes the lengths, also where no token can stay)
  const int most = a.budget < a.max_len ? a.budget : a.max_len;
  const long long pieces = (long long)most * (a.row_bytes / 16), each = 256 * kEvictPieces;
  const dim3 grid(pieces > each ? (unsigned)((pieces + each - 1) / each) : 1u, a.R);
  if (spread) hipLaunchKernelGGL(k_evict_move<true>, grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL(k_evict_move<false>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace up
