// Causal attention of a packed batch on the gfx950 matrix cores (Eq. 2's weights applied to the values), with the
// rows' log-sum-exp.
//
// One pass over the keys with a running softmax: for a row with reference m (log2 units), sum l and
// accumulator o, a tile of keys adds  l += sum_i 2^(x_i - m),  o += sum_i 2^(x_i - m) v_i  with
// x_i = scale*log2(e)*<q, k_i>; when a tile's maximum passes m by more than 2^8 the reference moves
// up and l, o are scaled down (any reference is exact; the margin spares most of the scalings).
//
// Work decomposition: a work-group is 8 (or 4) waves x 32 rows.  A row is a (token, query head) pair of one kv
// head, token-major, so the query heads that share keys share a tile and a single token is a small
// batch too.  Keys and values pass through LDS in tiles of 64 (32 where a head row has 512 bytes), two tiles at a time with eight waves,
// double-buffered, and loaded into it directly while the ones before them are worked on.  (Fetched into registers and written to LDS from there, with
// 128 rows per work-group: 9.31 ms for a prompt of 32768, 32/8 heads of 128; so 7.77 ms, 1.13 PFLOP/s.)
//
// The products are formed transposed: S^T = K Q^T leaves a lane with one query row and half of the
// tile's keys, so the softmax statistics are sums inside a lane and one exchange between lane
// halves, and the weights already sit in the operand layout of O^T = V^T P^T: the contraction runs over
// the keys in the order in which the lanes hold them.  V^T comes out of row-major LDS through the
// transposing read (bf16) or plain reads (float operands).
//
// Bound by the matrix cores and the vector work between their products at the clock that the power leaves (counters: a prompt of 32768,
// 128 wide, has the matrix cores busy in 57 % of the cycles and the vector pipe in 48 % at 1.76 GHz; 64 wide 53 and 83 % at 1.63 GHz:
// as many weights for half the products; a library's product of 8192^3 reaches 1.38 PFLOP/s); decode rows and short
// chunks on long caches by the latency of a work-group's tiles, which is why their keys are cut.
//
// Windowed (WINDOW): the same walk over the sinks and the band of keys that a tile's rows see, the stages that need no masks first.  A prompt of 32768,
// window 4096 and 128 sinks: 1.97-2.15 ms from one card to another, 0.99-1.08 PFLOP/s of the products that are seen (5 % more are walked over); one new
// token of 64 sequences, window 4096: 154 us, 5.2 TB/s; of one sequence, window 1024: 12 us, pieces of 128 keys and their join.  64 wide, window 1000,
// ragged and paged: 394-428 us, 0.57-0.62 PFLOP/s.  Of the 18 stages that a work-group walks over there 12 go without masks; 6 go with them, their pages
// looked up lane by lane: the 4 at the band's ends, and 2 that are whole and left over, as the loop without masks goes in pairs and stages ahead.  The
// masked stages of 64-wide bf16 heads read back 16 to 22 spilled registers (4 waves per SIMD leave 128).
//
// The weights enter the second product in bf16, their sum l in float.  Both other ways were measured, on the same inputs, as time and as
// the output's error against 64 bits (a prompt of 32768; 46290 tokens 64 wide; 16384 tokens 256 wide), with torch in float at 1.65e-3, 1.10e-3, 1.13e-3:
//   so                                             7.83 ms 1.91e-3     3.34 ms 1.19e-3     1.98 ms 1.23e-3
//   divided by the sum of the rounded weights      8.12 ms 1.73e-3     3.51 ms 1.12e-3     2.22 ms 1.15e-3
//   each weight in two bf16 parts, two products   10.73 ms 1.64e-3     4.71 ms 1.10e-3     2.70 ms 1.13e-3
// (most of an error is the output's own rounding).
#include <type_traits>

#include "up_attn.h"

namespace up {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

constexpr float kAttnSlack = 8.0f;      // log2 units by which a weight may pass 1 before the reference moves

template <bool F32, int D, int WAVES>
struct AttnTile {
  static constexpr int THREADS = 64 * WAVES, ROWS = 32 * WAVES;
  static constexpr int SRCB = D * (F32 ? 4 : 2);          // bytes of a head row
  static constexpr int PPR = SRCB / 16;                   // 16-byte pieces of it
  static constexpr int KT = SRCB == 512 ? 32 : 64;        // keys per tile
  static constexpr int SUB = KT / 32;
  static constexpr int TILES = WAVES == 8 ? 2 : 1;        // tiles staged at a time
  static constexpr int KS = KT * TILES;
  static_assert(KS == attn_stage_keys(SRCB, ROWS), "what the host counts with");
  static constexpr int PIECES = KS * PPR / THREADS;       // pieces per thread and staging
  static constexpr int ROWSTEP = THREADS / PPR;
  static constexpr int KREG = SRCB / 32;                  // 16-byte registers of a lane's half row
  static constexpr int DT = D / 32;
  // waves per SIMD that the registers are held to
  static constexpr int DENSE = SRCB == 128 ? 4 : SRCB == 512 && WAVES == 4 ? 1 : 2;
};

// Rows in LDS are not padded; the 16-byte pieces of a row are permuted instead (piece p sits in place p ^ swap(row)).
// Keys: 16 lanes that read the same piece of consecutive rows find 16 different places.  Values (bf16): the transposing
// read takes 64 bytes of 4 consecutive rows at a time.
template <int PPR>
__device__ __forceinline__ int k_swap(int row) { return row & (PPR < 16 ? PPR - 1 : 15); }
template <int PPR, bool F32>
__device__ __forceinline__ int v_swap(int row) { return F32 ? 0 : PPR == 8 ? (row & 2) << 1 : (row & 3) << 2; }
template <int PPR>
__device__ __forceinline__ int k_place(int row, int piece) { return row * PPR + (piece ^ k_swap<PPR>(row)); }
template <int PPR, bool F32>
__device__ __forceinline__ int v_place(int row, int piece) { return row * PPR + (piece ^ v_swap<PPR, F32>(row)); }

__device__ __forceinline__ float attn_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// (by value: a bit cast straight from an element of a vector takes the vector's first)
__device__ __forceinline__ float as_float(unsigned w) { return __builtin_bit_cast(float, w); }

// The value of the other lane half beside the own one: v_permlane32_swap exchanges the upper half of one register
// with the lower half of another, so of two copies one ends with the lower half's values everywhere, the other
// with the upper half's.
__device__ __forceinline__ f32x2 both_halves(float x) {
  const unsigned w = __builtin_bit_cast(unsigned, x);
  const auto r = __builtin_amdgcn_permlane32_swap(w, w, false, false);
  return f32x2{as_float(r[0]), as_float(r[1])};
}
__device__ __forceinline__ float half_max(float x) {
  const f32x2 v = both_halves(x);
  return fmaxf(v.x, v.y);
}
__device__ __forceinline__ float half_sum(float x) {
  const f32x2 v = both_halves(x);
  return v.x + v.y;
}

__device__ __forceinline__ unsigned pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

// Largest r with its first row tile at or before `slot` (the numbering of row tiles that needs no
// prefix sums: sequence r starts at slot cu[r] * Gq / rows + r).
__device__ __forceinline__ long long attn_slot_base(const AttnArgs& a, int r) { return (long long)a.cu[r] * a.Gq / a.rows + r; }
__device__ __forceinline__ int attn_slot_sequence(const AttnArgs& a, int slot) {
  int lo = 0, hi = a.R - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (attn_slot_base(a, mid) <= slot) lo = mid; else hi = mid - 1;
  }
  return lo;
}

struct AttnItem {
  int r;
  int tile, part;
  long long piece;      // number of the piece in the workspace, -1: the tile is not cut
};

// Windowed attention (WINDOW): the keys that a row tile sees are the sinks and a band.  The tile walks over them on an axis of its
// own: `sinks` places for the first keys (a whole number of stages; 0 where the band begins among them), then the band from key `low` on
// (a multiple of 8, so that the rows of a load stay within a page).
struct AttnBand {
  int sinks, low;
};
__device__ __forceinline__ AttnBand attn_band(const AttnArgs& a, int pos0) {
  const int first = pos0 - a.window + 1;                        // first key in the first row's window
  return first <= a.sinks ? AttnBand{0, 0} : AttnBand{a.sinks, first & ~7};
}
// keys (places) that a sequence's tiles walk over at most
template <bool WINDOW>
__device__ __forceinline__ int attn_reach(const AttnArgs& a, int Lk) { return WINDOW ? imin(Lk, a.reach) : Lk; }

// Length of sequence r where the lengths are on the device (one new token each)
__device__ __forceinline__ int attn_step_keys(const AttnArgs& a, int r) { return imax(0, imin(a.kv_len[r], a.max_len)); }

// Work item -> sequence, row tile, piece.  Unsplit launches number the row tiles without a prefix sum
// (a few numbers stand for nothing); split launches walk over the sequences' counts, 256 at a time.
template <int WAVES, bool SPLIT, bool WINDOW>
__device__ __forceinline__ bool attn_locate(const AttnArgs& a, int item, AttnItem& w, long long* sm) {
  constexpr int THREADS = 64 * WAVES, ROWS = 32 * WAVES;
  if (WINDOW && a.kv_len != nullptr) {      // one new token each: a.parts pieces of every sequence
    w.r = item / a.parts;
    w.part = item % a.parts;
    w.tile = 0;
    w.piece = SPLIT ? item : -1;
    return true;
  }
  if (!SPLIT) {
    w.r = attn_slot_sequence(a, item);
    w.tile = item - (int)attn_slot_base(a, w.r);
    w.part = 0;
    w.piece = -1;
    return (long long)w.tile * ROWS < (long long)(a.cu[w.r + 1] - a.cu[w.r]) * a.Gq;
  }
  // sm[0 .. WAVES): the waves' item sums, the WAVES after them: their piece sums, then the answer
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  long long* answer = sm + 2 * WAVES;
  long long items_before = 0, pieces_before = 0;
  for (int r0 = 0; r0 < a.R; r0 += THREADS) {
    const int r = r0 + tid;
    long long ni = 0, np = 0;
    int parts = 1;
    if (r < a.R) {
      const long long N = a.cu[r + 1] - a.cu[r];
      const long long tiles = (N * a.Gq + ROWS - 1) / ROWS;
      parts = attn_pieces(attn_reach<WINDOW>(a, a.cu_k[r + 1] - a.cu_k[r]), a.part_keys);
      ni = tiles * parts;
      np = parts > 1 ? ni : 0;
    }
    long long si = ni, sp = np;      // inclusive sums over the wave, then over the work-group
    for (int d = 1; d < 64; d <<= 1) {
      const long long oi = __shfl_up(si, d), op = __shfl_up(sp, d);
      if (lane >= d) { si += oi; sp += op; }
    }
    if (lane == 63) { sm[wave] = si; sm[WAVES + wave] = sp; }
    __syncthreads();
    long long items_here = 0, pieces_here = 0;
    for (int w2 = 0; w2 < WAVES; ++w2) {
      if (w2 == wave) { si += items_here; sp += pieces_here; }
      items_here += sm[w2];
      pieces_here += sm[WAVES + w2];
    }
    const long long first = items_before + si - ni;
    if (ni > 0 && item >= first && item < first + ni) {
      answer[0] = r;
      answer[1] = item - first;
      answer[2] = parts;
      answer[3] = parts > 1 ? pieces_before + sp - np : -1;
    }
    items_before += items_here;
    pieces_before += pieces_here;
    __syncthreads();
    if (item < items_before) {
      w.r = (int)answer[0];
      const int at = (int)answer[1], n = (int)answer[2];
      w.tile = at / n;
      w.part = at % n;
      w.piece = answer[3] < 0 ? -1 : answer[3] + at;
      return true;
    }
  }
  return false;
}

template <bool F32, int D, int WAVES, bool PAGED, bool SPLIT, bool WINDOW>
__global__ __launch_bounds__(64 * WAVES, (AttnTile<F32, D, WAVES>::DENSE)) void k_attn(AttnArgs a) {
  typedef AttnTile<F32, D, WAVES> T;
  // (two variables per buffer, not one array of buffers: the compiler then knows that a load into one and reads of
  // another do not meet, and does not wait for the load before them)
  __shared__ __align__(16) u32x4 sk0[T::KS * T::PPR], sk1[T::KS * T::PPR], sv0[T::KS * T::PPR], sv1[T::KS * T::PPR];
  static_assert(sizeof(sk0) * 4 <= 160 * 1024, "LDS of one CU");
  __shared__ long long scan[2 * WAVES + 4];
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  // the kv head runs fastest: with eight heads each of the eight L2s serves the tiles of one head;
  // the last row tiles, which see the most keys, start first
  const int kvh = blockIdx.x % a.Hkv;
  AttnItem w;
  if (!attn_locate<WAVES, SPLIT, WINDOW>(a, a.items - 1 - (int)(blockIdx.x / a.Hkv), w, scan)) return;
  const bool step = WINDOW && a.kv_len != nullptr;
  const int c0 = step ? w.r : a.cu[w.r], N = step ? 1 : a.cu[w.r + 1] - c0;
  const int ck0 = step ? 0 : a.cu_k[w.r], Lk = step ? attn_step_keys(a, w.r) : a.cu_k[w.r + 1] - ck0;
  if (step && Lk == 0) {      // nothing is seen: zeros, and the logarithm of nothing
    if (w.part != 0) return;
    if (SPLIT && kvh == 0 && tid == 0) a.base[w.r] = -1;
    char* dst = a.out + (long long)w.r * a.out_stride_b + (long long)kvh * a.Gq * T::SRCB;
    for (int i = tid; i < a.Gq * T::PPR; i += T::THREADS) ((u32x4*)dst)[i] = u32x4{0, 0, 0, 0};
    if (a.lse != nullptr && tid < a.Gq) a.lse[(long long)(kvh * a.Gq + tid) * a.lse_stride + w.r] = -INFINITY;
    return;
  }
  const long long row0 = (long long)w.tile * T::ROWS;
  const long long rows_left = (long long)N * a.Gq - row0;
  const int nrow = rows_left < T::ROWS ? (int)rows_left : T::ROWS;
  const int tok0 = (int)(row0 / a.Gq), rem0 = (int)(row0 % a.Gq);
  const int pos0 = Lk - N + tok0;                                  // position of the first row's token
  const int last_pos = pos0 + (rem0 + nrow - 1) / a.Gq;
  const AttnBand band = WINDOW ? attn_band(a, pos0) : AttnBand{0, 0};
  const int visible = band.sinks + last_pos + 1 - band.low;        // keys that the last row sees (places of the tile's axis)
  const int band_first = WINDOW ? imax(0, pos0 - a.window + 1) : 0;
  auto key_at = [&](int place) { return WINDOW && place >= band.sinks ? place - band.sinks + band.low : place; };
  const int k_begin = SPLIT ? w.part * a.part_keys : 0;
  const int k_end = SPLIT && a.part_keys < visible - k_begin ? k_begin + a.part_keys : visible;
  if (SPLIT && kvh == 0 && w.part == 0 && tid == 0)
    a.base[step ? w.r : attn_slot_base(a, w.r) + w.tile] = w.piece < 0 ? -1 : (int)w.piece;
  if (k_begin >= visible) return;

  // ---- this lane's row
  const int uwave = __builtin_amdgcn_readfirstlane(wave);           // (uniform: branches on it are scalar)
  const bool wave_live = uwave * 32 < nrow;
  const int x = imin(wave * 32 + l32, nrow - 1);                   // (rows past the end repeat the last one)
  const int tok = (rem0 + x) / a.Gq, hh = (rem0 + x) % a.Gq;
  const int pos = pos0 + tok;
  const int wave_last = pos0 + (rem0 + imin(uwave * 32 + 31, nrow - 1)) / a.Gq;
  const int wave_first = pos0 + (rem0 + imin(uwave * 32, nrow - 1)) / a.Gq;
  constexpr int HOFF = F32 ? T::SRCB / 2 : 16, KSTEP = F32 ? 16 : 32;
  u32x4 qf[T::KREG];
  {
    const char* src = a.q + (long long)(c0 + tok0 + tok) * a.q_stride_b + (long long)(kvh * a.Gq + hh) * T::SRCB + half * HOFF;
#pragma unroll
    for (int kk = 0; kk < T::KREG; ++kk) qf[kk] = *(const u32x4*)(src + kk * KSTEP);
  }

  // ---- staging, straight from memory into LDS: a wave's load writes 64 consecutive 16-byte places, WROWS rows,
  // lane l the place l % PPR of row l / PPR; the permutation of a row's pieces is in the address that the lane reads.
  // Keys past the end repeat the last one (their weights are zero).  Where the rows of a load lie side by side
  // (packed keys, or pages of a multiple of 8 tokens) and before the end, its address is a scalar plus a constant per lane.
  constexpr int WROWS = 64 / T::PPR;
  const int lrow = lane / T::PPR, lplace = lane % T::PPR;
  const char* k_head = a.k + (long long)kvh * T::SRCB;
  const char* v_head = a.v + (long long)kvh * T::SRCB;
  // (rows of 512 bytes: the rows of a lane's loads are 8 apart, and the keys' permutation has period 16)
  const unsigned k_at[2] = {(unsigned)(lplace ^ k_swap<T::PPR>(uwave * WROWS + lrow)) * 16u,
                            (unsigned)(lplace ^ k_swap<T::PPR>(T::ROWSTEP + uwave * WROWS + lrow)) * 16u};
  const unsigned v_at = (unsigned)(lplace ^ v_swap<T::PPR, F32>(uwave * WROWS + lrow)) * 16u;
  const unsigned k_lane[2] = {(unsigned)lrow * (unsigned)a.k_stride_b + k_at[0], (unsigned)lrow * (unsigned)a.k_stride_b + k_at[1]};
  const unsigned v_lane = (unsigned)lrow * (unsigned)a.v_stride_b + v_at;
  const bool in_runs = !PAGED || (a.kv_block & 7) == 0;
  const int32_t* table = PAGED ? a.block_table + (long long)w.r * a.table_stride : nullptr;
  auto row_of = [&](int key) -> long long {
    if (!PAGED) return (long long)ck0 + key;
    unsigned blk, at;
    divmod_by((unsigned)key, (unsigned)a.kv_block, a.kv_magic, blk, at);
    return (long long)table[blk] * a.kv_block + at;
  };
  auto stage_run = [&](int k0, u32x4* sk, u32x4* sv) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < T::PIECES; ++i) {
      const int r0 = i * T::ROWSTEP + uwave * WROWS;
      long long row = (long long)ck0 + k0 + r0;
      if (PAGED) {
        unsigned blk, at;
        divmod_by((unsigned)(k0 + r0), (unsigned)a.kv_block, a.kv_magic, blk, at);
        row = (long long)table_entry(table, blk) * a.kv_block + at;
      }
      load_to_lds(k_head + row * a.k_stride_b + k_lane[i & 1], sk + r0 * T::PPR);
      load_to_lds(v_head + row * a.v_stride_b + v_lane, sv + r0 * T::PPR);
    }
  };
  auto stage_any = [&](int k0, u32x4* sk, u32x4* sv) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < T::PIECES; ++i) {
      const int r0 = i * T::ROWSTEP + uwave * WROWS;
      int key = imin(k0 + r0 + lrow, Lk - 1);
      if (WINDOW && key >= a.n_sink && key < band_first) key = band_first;      // (what no row sees is not read: its page may be gone)
      const long long row = row_of(key);
      load_to_lds(k_head + row * a.k_stride_b + k_at[i & 1], sk + r0 * T::PPR);
      load_to_lds(v_head + row * a.v_stride_b + v_at, sv + r0 * T::PPR);
    }
  };

  f32x16 o[T::DT];
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[dt][e] = 0.0f;
  float m = -INFINITY, l = 0.0f;

  // The permuted place of piece p is that of piece 0 with p's bits turned over, so a lane's addresses are one constant and an exclusive or
  // each.  For 512-byte rows the constant is made anew in every tile: kept over the loop, the addresses pushed accumulators into
  // scratch (72 registers of it, 4.84 ms for a prompt of 16384 with 16 heads; now 25 and 1.98 ms).
  // mask_tag: some keys of the tile come after some rows of the wave.
  auto tile = [&](auto mask_tag, int k0, const u32x4* sk, const u32x4* sv) __attribute__((always_inline)) {
    unsigned k_from = (unsigned)k_place<T::PPR>(l32, F32 ? half * (T::PPR / 2) : half) * 16u;
    if constexpr (T::SRCB == 512) asm volatile("" : "+v"(k_from));
    f32x16 s[T::SUB];
#pragma unroll
    for (int sub = 0; sub < T::SUB; ++sub) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[sub][e] = 0.0f;
#pragma unroll
      for (int kk = 0; kk < T::KREG; ++kk) {
        const u32x4 k4 = *(const u32x4*)((const char*)sk + (k_from ^ (unsigned)(kk * KSTEP)) + sub * 32 * T::SRCB);
        if (F32) {
          const u32x4 q4 = qf[kk];
#pragma unroll
          for (int i = 0; i < 4; ++i) s[sub] = __builtin_amdgcn_mfma_f32_32x32x2f32(as_float(k4[i]), as_float(q4[i]), s[sub], 0, 0, 0);
        } else {
          s[sub] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, k4), __builtin_bit_cast(bf16x8, qf[kk]), s[sub], 0, 0, 0);
        }
      }
    }
    // element e of s[sub]: key k0 + 32*sub + 8*(e/4) + 4*half + e%4, row l32
    if (decltype(mask_tag)::value) {
      const int ago = pos - k0 - 4 * half;      // how far the row is past the lane's first key
      if (!WINDOW || k0 < a.n_sink) {
#pragma unroll
        for (int sub = 0; sub < T::SUB; ++sub)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = sub * 32 + 8 * (e >> 2) + (e & 3);
            if (WINDOW ? ago < at || (ago - at >= a.window && k0 + 4 * half + at >= a.n_sink) : k0 + at + 4 * half > pos) s[sub][e] = -INFINITY;
          }
      } else {      // (one comparison for both ends of a window, in unsigned numbers)
#pragma unroll
        for (int sub = 0; sub < T::SUB; ++sub)
#pragma unroll
          for (int e = 0; e < 16; ++e)
            if ((unsigned)(ago - (sub * 32 + 8 * (e >> 2) + (e & 3))) >= (unsigned)a.window) s[sub][e] = -INFINITY;
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int sub = 0; sub < T::SUB; ++sub)
#pragma unroll
      for (int e = 0; e < 16; e += 8) {
        float m8 = fmaxf(fmaxf(s[sub][e], s[sub][e + 1]), s[sub][e + 2]);
        m8 = fmaxf(fmaxf(m8, s[sub][e + 3]), s[sub][e + 4]);
        m8 = fmaxf(fmaxf(m8, s[sub][e + 5]), s[sub][e + 6]);
        mx = fmaxf(fmaxf(m8, s[sub][e + 7]), mx);
      }
    const float ref = half_max(mx) * a.c;
    if (__any(ref > m + kAttnSlack)) {
      const float up = fmaxf(m, ref);
      const float f = m == -INFINITY ? 0.0f : attn_exp2(m - up);
      m = up;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= f;
    }
    const float neg = m == -INFINITY ? 0.0f : -m;      // (a row that has seen no key yet: all weights 2^-inf)
    float l0 = 0.0f, l1 = 0.0f;
#pragma unroll
    for (int sub = 0; sub < T::SUB; ++sub)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        s[sub][e] = attn_exp2(fmaf(s[sub][e], a.c, neg));
        s[sub][e + 1] = attn_exp2(fmaf(s[sub][e + 1], a.c, neg));
        l0 += s[sub][e];
        l1 += s[sub][e + 1];
      }
    l += l0 + l1;
    // (Rows of 128 bytes, four waves to a SIMD: the wave that has its weights goes first, and the others' exponentials fill in; 46290
    // tokens in seven sequences 3.41 -> 3.35 ms.  Two waves lose by it: 128 wide, paged, 8.01 -> 8.18 ms.)
    if constexpr (T::SRCB == 128) __builtin_amdgcn_s_setprio(1);
    // O^T += V^T P^T.  A contraction step takes keys in the order the lanes hold their weights.
    if (F32) {
#pragma unroll
      for (int sub = 0; sub < T::SUB; ++sub)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int row = sub * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
#pragma unroll
          for (int dt = 0; dt < T::DT; ++dt) {
            const float v = ((const float*)sv)[row * D + dt * 32 + l32];
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x2f32(v, s[sub][e], o[dt], 0, 0, 0);
          }
        }
    } else {
      // 16 keys per step: lane half h holds keys 4h..4h+3 and 8+4h..8+4h+3 of them.  The transposing
      // read gives 16 lanes a column each of 4 rows x 16 columns: its lane i points at row i/4, columns 4*(i%4)..
      const int vrow = 4 * half + ((lane >> 2) & 3);
      const int vpc = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1), vlo = (lane & 1) * 8;
      unsigned v_from = (unsigned)v_place<T::PPR, F32>(vrow, vpc) * 16u + vlo;
      if constexpr (T::SRCB == 512) asm volatile("" : "+v"(v_from));
      // columns 32*dt.. of keys `row`.. of the tile.  (Rows of 256 bytes and fewer are indexed plainly: with the exclusive or, the
      // 128-wide kernel came out 1.2 % slower, 7.88 against 7.79 ms for a prompt of 32768.)
      auto v_at = [&](int row, int dt) __attribute__((always_inline)) {
        if constexpr (T::SRCB == 512) return (const char*)sv + (v_from ^ (unsigned)(dt * 64)) + row * T::SRCB;
        else return (const char*)&sv[v_place<T::PPR, F32>(row + vrow, dt * 4 + vpc)] + vlo;
      };
#pragma unroll
      for (int sub = 0; sub < T::SUB; ++sub)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          u32x4 pw;
          pw.x = pack_bf16(s[sub][8 * st], s[sub][8 * st + 1]);
          pw.y = pack_bf16(s[sub][8 * st + 2], s[sub][8 * st + 3]);
          pw.z = pack_bf16(s[sub][8 * st + 4], s[sub][8 * st + 5]);
          pw.w = pack_bf16(s[sub][8 * st + 6], s[sub][8 * st + 7]);
#pragma unroll
          for (int dt = 0; dt < T::DT; ++dt) {
            const int row = sub * 32 + st * 16;
            typedef __attribute__((address_space(3))) s16x4* lds4;
            const s16x4 va = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(__attribute__((address_space(3))) char*)v_at(row, dt));
            const s16x4 vb = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(__attribute__((address_space(3))) char*)v_at(row + 8, dt));
            u32x4 vv;
            vv.x = __builtin_bit_cast(u32x2, va).x;
            vv.y = __builtin_bit_cast(u32x2, va).y;
            vv.z = __builtin_bit_cast(u32x2, vb).x;
            vv.w = __builtin_bit_cast(u32x2, vb).y;
            o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vv), __builtin_bit_cast(bf16x8, pw), o[dt], 0, 0, 0);
          }
        }
    }
    if constexpr (T::SRCB == 128) __builtin_amdgcn_s_setprio(0);
  };

  // Tiles that every row sees whole and whose successor lies before the end first; then the few at the
  // end that need the masks (or, for pages of other sizes, all of them).
  auto staged = [&]() {      // the next tile is in LDS and everyone is done with this one
    __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    __syncthreads();
  };
  // (tiles are staged while the ones before them are worked on; the last readers of their buffer passed a barrier)
  constexpr int NEXT = T::KT * T::PPR;      // places of a tile in LDS
  auto whole_tiles = [&](int k0, const u32x4* sk, const u32x4* sv) __attribute__((always_inline)) {
    if (!wave_live) return;
#pragma unroll
    for (int u = 0; u < T::TILES; ++u) tile(std::false_type{}, k0 + u * T::KT, sk + u * NEXT, sv + u * NEXT);
  };
  auto last_tiles = [&](int k0, const u32x4* sk, const u32x4* sv) __attribute__((always_inline)) {
    if (!wave_live) return;
    for (int u = 0; u < T::TILES; ++u) {
      const int key = key_at(k0) + u * T::KT;
      if (WINDOW && key >= a.n_sink && key + T::KT - 1 <= wave_first - a.window) continue;      // all before the wave's windows
      if (key <= wave_last && k0 + u * T::KT < k_end) tile(std::true_type{}, key, sk + u * NEXT, sv + u * NEXT);
    }
  };
  if constexpr (WINDOW) {
    // Stages that every row sees whole lie among the sinks ([s0, s1)) and in the middle of the band ([s2, s3)); the sums do not ask for
    // an order, so these come first, as q = 0 .. n_whole - 1, and the stages that need the masks after them.  (In one loop that chose
    // between the two ways to stage, and between masks and none, the registers of the 256-wide kernel spilled 800 times, 2297 us for a
    // prompt of 32768 with a window of 4096 against 1965; and where the two ways of a stage ended in the same loads, the
    // listing had one of them load from registers that nothing had set on that way; that form was never run, nor its cause found.)
    const int first = k_begin / T::KS, last = (k_end + T::KS - 1) / T::KS;
    auto within = [&](int place) { return imax(first, imin(last, place / T::KS)); };
    const int band_whole = band.sinks + imax(0, last_pos - a.window + 1 - band.low + T::KS - 1);      // (rounded up: places from here on are in every window)
    const int s1 = within(imin(a.n_sink, pos0 + 1)), s2 = imax(s1, within(band_whole));
    const int s3 = imax(s2, within(imin(k_end, band.sinks + pos0 + 1 - band.low)));
    const int n_sinks = s1 - first, n_whole = n_sinks + s3 - s2;
    auto place_of = [&](int q) {
      const int i = q - n_whole, s = q < n_sinks ? first + q : q < n_whole ? s2 + q - n_sinks : i < s2 - s1 ? s1 + i : s3 + i - (s2 - s1);
      return s * T::KS;
    };
    const int n = last - first;
    stage_any(key_at(place_of(0)), sk0, sv0);
    staged();
    int q = 0;
    if (in_runs) {
      for (; q + 2 < n_whole; q += 2) {
        stage_run(key_at(place_of(q + 1)), sk1, sv1);
        whole_tiles(key_at(place_of(q)), sk0, sv0);
        staged();
        stage_run(key_at(place_of(q + 2)), sk0, sv0);
        whole_tiles(key_at(place_of(q + 1)), sk1, sv1);
        staged();
      }
    }
    for (; q < n; q += 2) {
      if (q + 1 < n) stage_any(key_at(place_of(q + 1)), sk1, sv1);
      last_tiles(place_of(q), sk0, sv0);
      staged();
      if (q + 1 >= n) break;
      if (q + 2 < n) stage_any(key_at(place_of(q + 2)), sk0, sv0);
      last_tiles(place_of(q + 1), sk1, sv1);
      staged();
    }
  } else {
  stage_any(k_begin, sk0, sv0);
  staged();
  int k0 = k_begin;
  const int whole = in_runs ? imin(imin(k_end, pos0 + 1), Lk - T::KS) - T::KS : k_begin - 1;
  for (; k0 + T::KS <= whole; k0 += 2 * T::KS) {
    stage_run(k0 + T::KS, sk1, sv1);
    whole_tiles(k0, sk0, sv0);
    staged();
    stage_run(k0 + 2 * T::KS, sk0, sv0);
    whole_tiles(k0 + T::KS, sk1, sv1);
    staged();
  }
  for (; k0 < k_end; k0 += 2 * T::KS) {
    if (k0 + T::KS < k_end) stage_any(k0 + T::KS, sk1, sv1);
    last_tiles(k0, sk0, sv0);
    staged();
    if (k0 + T::KS >= k_end) break;
    if (k0 + 2 * T::KS < k_end) stage_any(k0 + 2 * T::KS, sk0, sv0);
    last_tiles(k0 + T::KS, sk1, sv1);
    staged();
  }
  }

  l = half_sum(l);
  if (!wave_live || wave * 32 + l32 >= nrow) return;
  const int t = c0 + tok0 + tok, h = kvh * a.Gq + hh;
  if (SPLIT && w.piece >= 0) {
    const long long at = (w.piece * a.Hkv + kvh) * T::ROWS + x;
    float* dst = a.o_part + at * D;
#pragma unroll
    for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *(f32x4*)(dst + dt * 32 + 8 * j + 4 * half) = f32x4{o[dt][4 * j], o[dt][4 * j + 1], o[dt][4 * j + 2], o[dt][4 * j + 3]};
    if (half == 0) {
      a.ml_part[2 * at] = m;
      a.ml_part[2 * at + 1] = l;
    }
    return;
  }
  const float inv = 1.0f / l;
  char* dst = a.out + (long long)t * a.out_stride_b + (long long)h * T::SRCB;
#pragma unroll
  for (int dt = 0; dt < T::DT; ++dt)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int d = dt * 32 + 8 * j + 4 * half;
      const float v0 = o[dt][4 * j] * inv, v1 = o[dt][4 * j + 1] * inv, v2 = o[dt][4 * j + 2] * inv, v3 = o[dt][4 * j + 3] * inv;
      if (F32) *(f32x4*)(dst + d * 4) = f32x4{v0, v1, v2, v3};
      else *(u32x2*)(dst + d * 2) = u32x2{pack_bf16(v0, v1), pack_bf16(v2, v3)};
    }
  if (a.lse != nullptr && half == 0) a.lse[(long long)h * a.lse_stride + t] = (m + __log2f(l)) * 0.69314718055994530942f;
}

// Joins the pieces of the row tiles that were cut: a wave per row, the pieces in order.
template <bool F32, int D, bool WINDOW>
__global__ __launch_bounds__(256) void k_attn_join(AttnArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int kvh = blockIdx.x % a.Hkv, slot = blockIdx.x / a.Hkv;
  const bool step = WINDOW && a.kv_len != nullptr;
  const int r = step ? slot : attn_slot_sequence(a, slot), c0 = step ? r : a.cu[r], N = step ? 1 : a.cu[r + 1] - c0;
  const int Lk = step ? attn_step_keys(a, r) : a.cu_k[r + 1] - a.cu_k[r];
  const int tile = step ? 0 : slot - (int)attn_slot_base(a, r);
  const long long row0 = (long long)tile * a.rows, rows_left = (long long)N * a.Gq - row0;
  if (rows_left <= 0) return;
  const int first = a.base[slot];
  if (first < 0) return;
  const int nrow = rows_left < a.rows ? (int)rows_left : a.rows;
  const int tok0 = (int)(row0 / a.Gq), rem0 = (int)(row0 % a.Gq);
  const AttnBand band = WINDOW ? attn_band(a, Lk - N + tok0) : AttnBand{0, 0};
  const int visible = band.sinks + Lk - N + tok0 + (rem0 + nrow - 1) / a.Gq + 1 - band.low;
  const int parts = attn_pieces(visible, a.part_keys);      // pieces that saw a key
  constexpr int PER = D / 64;
  for (int x = blockIdx.y * 4 + wave; x < nrow; x += gridDim.y * 4) {
    const long long step = (long long)a.Hkv * a.rows, at0 = ((long long)first * a.Hkv + kvh) * a.rows + x;
    float m = -INFINITY;
    for (int p = 0; p < parts; ++p) m = fmaxf(m, a.ml_part[2 * (at0 + p * step)]);
    float l = 0.0f, acc[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = 0.0f;
    for (int p = 0; p < parts; ++p) {
      const long long at = at0 + p * step;
      const float mp = a.ml_part[2 * at];
      const float f = mp == -INFINITY ? 0.0f : attn_exp2(mp - m);
      l = fmaf(a.ml_part[2 * at + 1], f, l);
#pragma unroll
      for (int i = 0; i < PER; ++i) acc[i] = fmaf(a.o_part[at * D + lane * PER + i], f, acc[i]);
    }
    const int t = c0 + tok0 + (rem0 + x) / a.Gq, h = kvh * a.Gq + (rem0 + x) % a.Gq;
    const float inv = 1.0f / l;
    char* dst = a.out + (long long)t * a.out_stride_b + (long long)h * D * (F32 ? 4 : 2);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (F32) ((float*)dst)[lane * PER + i] = acc[i] * inv;
      else ((__bf16*)dst)[lane * PER + i] = (__bf16)(acc[i] * inv);
    }
    if (a.lse != nullptr && lane == 0) a.lse[(long long)h * a.lse_stride + t] = (m + __log2f(l)) * 0.69314718055994530942f;
  }
}

template <bool F32, int D, int WAVES, bool PAGED, bool WINDOW>
static hipError_t launch_attn(const AttnArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.items * a.Hkv), block(64 * WAVES);
  if (a.part_keys == 0) {
    hipLaunchKernelGGL((k_attn<F32, D, WAVES, PAGED, false, WINDOW>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((k_attn<F32, D, WAVES, PAGED, true, WINDOW>), grid, block, 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((k_attn_join<F32, D, WINDOW>), dim3((unsigned)a.slots * a.Hkv, 8), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <bool F32, int D, bool PAGED>
static hipError_t launch_attn_rows(const AttnArgs& a, hipStream_t s) {
  if (a.window > 0) return a.rows == 256 ? launch_attn<F32, D, 8, PAGED, true>(a, s) : launch_attn<F32, D, 4, PAGED, true>(a, s);
  return a.rows == 256 ? launch_attn<F32, D, 8, PAGED, false>(a, s) : launch_attn<F32, D, 4, PAGED, false>(a, s);
}

template <bool F32, int D>
static hipError_t launch_attn_form(const AttnArgs& a, hipStream_t s) {
  return a.block_table != nullptr ? launch_attn_rows<F32, D, true>(a, s) : launch_attn_rows<F32, D, false>(a, s);
}

hipError_t launch_attention(const AttnArgs& a, bool f32, int D, hipStream_t s) {
  if (f32) return D == 64 ? launch_attn_form<true, 64>(a, s) : launch_attn_form<true, 128>(a, s);
  return D == 64 ? launch_attn_form<false, 64>(a, s) : D == 128 ? launch_attn_form<false, 128>(a, s) : launch_attn_form<false, 256>(a, s);
}

}  // namespace up
