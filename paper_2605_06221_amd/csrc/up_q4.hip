// The 4-bit KV cache: rows into it and out of it, and the decode attention over it.
//
// An element stands for lo + step * code with one (lo, step) pair of bf16 per 64 elements of a head
// row (4.5 bits per element).  The attention never forms those values: codes are whole numbers, exact
// in bf16, so the matrix cores multiply codes and the pairs enter in float,
//     <q, k_i>      = sum_g step_g,i (q_g . c_g,i) + lo_g,i (sum of q_g),
//     sum_i w_i v_i = sum_i (w_i step_g,i) c_g,i + sum_i w_i lo_g,i.
#include "up_attn.h"

namespace up {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

namespace {

template <int CTRL>
__device__ __forceinline__ float lane_dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ unsigned pack2(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

// (by value: a bit cast straight from an element of a vector takes the vector's first)
__device__ __forceinline__ float word_float(unsigned w) { return __builtin_bit_cast(float, w); }

// bits of the largest bf16 not above x, in the upper half of the word
__device__ __forceinline__ unsigned bf16_below(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x);
  return (b >> 31 ? b + 0xffffu : b) & 0xffff0000u;
}
// Bits of the smallest bf16 not below (mx - lo) / 15.  A bf16 times 15 is exact, so the comparison decides the quotient without a
// division.  In float, with the range as a sum of two floats, its estimate taken a little too large so that truncated to bf16 it is the
// answer or the bf16 below; in double for ranges near the ends of the float range (and 0).
__device__ __forceinline__ unsigned step_of(float mx, float lo) {
  const float r = mx - lo;
  if (r > 1e-30f && r < 1e30f) {
    const float back = r - mx, rest = (mx - (r - back)) - (lo + back);      // r + rest = mx - lo
    const unsigned b = __builtin_bit_cast(unsigned, r * (1.000001f / 15.0f)) & 0xffff0000u;
    const float p = 15.0f * word_float(b);
    return p > r || (p == r && rest <= 0.0f) ? b : b + 0x10000u;
  }
  const double range = (double)mx - (double)lo;
  unsigned b = __builtin_bit_cast(unsigned, (float)(range * (1.0 / 15.0))) & 0xffff0000u;
  if (b > 0 && 15.0 * (double)word_float(b - 0x10000u) >= range) b -= 0x10000u;
  else if (15.0 * (double)word_float(b) < range) b += 0x10000u;
  return b;
}

// LANES lanes hold the 64 elements of a group.  The groups of all rows stand in a row; a work-group takes UNITS x 256 / LANES of
// them of the keys (blockIdx.y 0) or of the values, and every thread issues the loads of its UNITS before it looks at one.
constexpr int kQ4Block = 128;      // groups per work-group
struct Q4Unit { bool live; int64_t slot; int t, g; };
template <int LANES, int UNITS>
__device__ __forceinline__ void q4_units(const Q4CopyArgs& a, int groups, Q4Unit (&u)[UNITS]) {
  static_assert(UNITS * 256 / LANES == kQ4Block, "the launch's grid");
  const unsigned magic = 0xFFFFFFFFu / (unsigned)groups;
  const long long n = a.count_dev != nullptr && a.count_dev[0] < a.n ? a.count_dev[0] : a.n;
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    unsigned t, g;
    divmod_by((blockIdx.x * UNITS + i) * (256u / LANES) + threadIdx.x / LANES, (unsigned)groups, magic, t, g);
    u[i].t = (int)t;
    u[i].g = (int)g;
    u[i].live = (long long)t < n;
    u[i].slot = u[i].live ? a.slots[t] : -1;
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) u[i].live = u[i].slot >= 0 && u[i].slot < a.num_slots;
}

// A lane takes two pieces of eight elements, so that what is done once per group (its place, the reduction over the lanes, the step) is
// shared by sixteen.  (One piece per lane, eight lanes to a group, the step in double, and a branch for everything next to a tie, which some lane of
// nearly every wave takes: bound by its instructions, 179 us for the keys and values of 131072 tokens, 8 heads of 128; so 143 us,
// 4.8 TB/s, what a copy reaches.)
template <bool F32>
__global__ __launch_bounds__(256) void k_q4_store(Q4CopyArgs a) {
  constexpr int LANES = 4, UNITS = 2, PIECES = 2, PER = F32 ? 2 : 1;
  const int kv = blockIdx.y, sub = threadIdx.x & (LANES - 1);
  if (a.cache[kv] == nullptr) return;
  const int groups = a.heads * (a.D / kQ4Group);
  const long long codes = q4_code_bytes(a.heads, a.D);
  Q4Unit u[UNITS];
  q4_units<LANES, UNITS>(a, groups, u);
  u32x4 w[UNITS][PIECES][PER];
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    const char* src = a.rows_in[kv] + (long long)u[i].t * a.row_stride_b[kv] + (u[i].g * 8 + sub) * (F32 ? 32 : 16);
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int j = 0; j < PER; ++j)
        w[i][p][j] = u[i].live ? __builtin_nontemporal_load((const u32x4*)src + p * LANES * PER + j) : u32x4{0, 0, 0, 0};
  }
#pragma unroll
  for (int i = 0; i < UNITS; ++i) {
    float x[PIECES][8], mn = INFINITY, mx = -INFINITY, least = INFINITY;      // least: the smallest magnitude
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[p][2 * e] = F32 ? word_float(w[i][p][F32 ? e / 2 : 0][(2 * e) & 3]) : bf16_lo(w[i][p][0][e]);
        x[p][2 * e + 1] = F32 ? word_float(w[i][p][F32 ? e / 2 : 0][(2 * e + 1) & 3]) : bf16_hi(w[i][p][0][e]);
        mn = fminf(fminf(mn, x[p][2 * e]), x[p][2 * e + 1]);
        mx = fmaxf(fmaxf(mx, x[p][2 * e]), x[p][2 * e + 1]);
        if (!F32) least = fminf(fminf(least, fabsf(x[p][2 * e])), fabsf(x[p][2 * e + 1]));
      }
    }
    mn = fminf(mn, lane_dpp<0xB1>(mn)); mx = fmaxf(mx, lane_dpp<0xB1>(mx));
    mn = fminf(mn, lane_dpp<0x4E>(mn)); mx = fmaxf(mx, lane_dpp<0x4E>(mx));
    // (least stays the lane's: it is asked about the lane's elements)
    const unsigned lo_bits = bf16_below(mn);
    const float lo = word_float(lo_bits);
    const unsigned step_bits = step_of(mx, lo);
    const float step = word_float(step_bits);
    // A code is the quotient (x - lo) / step rounded to even, and one in 340 of normal bf16 elements is a true tie.  bf16: where neither lo
    // nor an element of the lane is below 2^-15 of the largest magnitude, x - lo is exact in float, a quotient that is
    // representable comes out exact after one correction, and one that is no tie keeps 2^-20.1 from it, more than its rounding
    // error, 2^-21.  Otherwise, and for float, a code is judged by what it leaves: rests next to half a step are looked at once more, in
    // double where x - lo was rounded; so are steps whose reciprocal or range leaves the float range.  (A code plus kWhole is
    // rounded to a whole number and sits in the float's low bits.)
    constexpr float kWhole = 12582912.0f;
    const float inv = __builtin_amdgcn_rcpf(step), half = 0.5f * step;
    float whole[PIECES][8], far = 0.0f;
#pragma unroll
    for (int p = 0; p < PIECES; ++p)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = x[p][e] - lo, q = d * inv;
        whole[p][e] = fmaf(fmaf(-q, step, d), inv, q) + kWhole;
        if (F32) far = fmaxf(far, fabsf(fmaf(kWhole - whole[p][e], step, d)));
      }
    const bool plain = step > 1e-25f && step < 1e30f;
    if (!F32 && lo != 0.0f) least = fminf(least, fabsf(lo));
    if (!plain || (F32 ? far > half * 0.99999f : least < fmaxf(fabsf(lo), fabsf(mx)) * 0x1p-15f)) {
#pragma unroll
      for (int p = 0; p < PIECES; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float d = x[p][e] - lo, rest = fmaf(kWhole - whole[p][e], step, d), off = fabsf(rest);
          if (plain && off <= half * 0.99999f) continue;
          if (plain && d + lo == x[p][e] && x[p][e] - d == lo) {
            const bool odd = __builtin_bit_cast(unsigned, whole[p][e]) & 1u;
            if (off > half || (off == half && odd)) whole[p][e] += rest > 0.0f ? 1.0f : -1.0f;
          } else {
            const double c = step > 0.0f ? rint(((double)x[p][e] - (double)lo) / (double)step) : 0.0;
            whole[p][e] = (float)fmin(fmax(c, 0.0), 15.0) + kWhole;
          }
        }
    }
    if (!u[i].live) continue;
    char* dst = a.cache[kv] + (long long)u[i].slot * a.cache_stride;
#pragma unroll
    for (int p = 0; p < PIECES; ++p) {
      // sum of bits(code + kWhole) << 4e: what kWhole's own bits add is known
      unsigned packed = __builtin_bit_cast(unsigned, whole[p][7]);
#pragma unroll
      for (int e = 6; e >= 0; --e) packed = (packed << 4) + __builtin_bit_cast(unsigned, whole[p][e]);
      packed -= 0x4B400000u + (0x4B400000u << 4) + (0x4B400000u << 8);
      *(unsigned*)(dst + u[i].g * 32 + (p * LANES + sub) * 4) = packed;
    }
    if (sub == 0) *(unsigned*)(dst + codes + (long long)u[i].g * 4) = (lo_bits >> 16) | step_bits;
  }
}

constexpr int kQ4Units = 4;
template <bool F32>
__global__ __launch_bounds__(256) void k_q4_load(Q4CopyArgs a) {
  const int kv = blockIdx.y, sub = threadIdx.x & 7;
  if (a.cache[kv] == nullptr) return;
  const int groups = a.heads * (a.D / kQ4Group);
  const long long codes = q4_code_bytes(a.heads, a.D);
  Q4Unit u[kQ4Units];
  q4_units<8, kQ4Units>(a, groups, u);
  unsigned packed[kQ4Units], pair[kQ4Units];
#pragma unroll
  for (int i = 0; i < kQ4Units; ++i) {
    const char* src = a.cache[kv] + (u[i].live ? u[i].slot : 0) * a.cache_stride;
    packed[i] = u[i].live ? *(const unsigned*)(src + u[i].g * 32 + sub * 4) : 0u;
    pair[i] = u[i].live ? *(const unsigned*)(src + codes + (long long)u[i].g * 4) : 0u;
  }
#pragma unroll
  for (int i = 0; i < kQ4Units; ++i) {
    if (!u[i].live) continue;
    const float lo = bf16_lo(pair[i]), step = bf16_hi(pair[i]);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = fmaf((float)((packed[i] >> (4 * e)) & 15u), step, lo);
    // bf16: rounding the float rounds the value itself once, for the float is exact or no bf16 number or middle between two lies
    // between them, but for a lo below step / 2^12, which a float may lose.  With 2^e the power of two at or below step, code * step is a
    // multiple of 2^(e-7), and where bf16 decides next to it are multiples of 2^(e-8) (below a power of two: of 2^(e-9)).  Any lo of
    // the same sign below 2^(e-9) then rounds alike, step / 2^10 among them, and with that one the float is exact.
    const float least = step * 0x1p-10f;
    if (!F32 && fabsf(lo) < least && lo != 0.0f) {
      const float lo2 = copysignf(least, lo);
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = x[e] == lo ? lo : fmaf((float)((packed[i] >> (4 * e)) & 15u), step, lo2);
    }
    char* dst = a.rows_out[kv] + (long long)u[i].t * a.row_stride_b[kv] + (u[i].g * 8 + sub) * (F32 ? 32 : 16);
    if (F32) {
      __builtin_nontemporal_store(f32x4{x[0], x[1], x[2], x[3]}, (f32x4*)dst);
      __builtin_nontemporal_store(f32x4{x[4], x[5], x[6], x[7]}, (f32x4*)dst + 1);
    } else {
      __builtin_nontemporal_store(u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])}, (u32x4*)dst);
    }
  }
}

// ---------------------------------------------------------------------------------------------------- decode
// A wave takes one kv head and 64 keys at a time, all by itself (no barriers):
//   S^T = C_k Q^T  in v_mfma_f32_16x16x32_bf16 tiles of 16 keys x 16 query heads, one accumulator per
//         group of 64 elements; lane = one query head and keys 16t + 4*quarter + j;
//   O^T = C_v^T P'^T with P' = weight * step, again one operand per group, rounded to bf16.  (P' in two bf16 parts and two products: 1000
//         cached tokens come out at an error of 1.63e-3, that of their own rounding, instead of 2.14e-3, longer caches hardly differ (1.66e-3 against
//         1.68e-3 for 48 ragged ones, 1.53e-3 both ways for 131072 tokens), and they take 134 instead of 129 us, 58 instead of 54.)
// Codes of eight keys sit in one word; a shift and (w & 0x00780078) | 0x41804180 make two bf16 numbers 16 + code
// (0x4180 = 16.0, whose mantissa has the code's place at bits 3..6), and the 16 goes into the lowest value: lo - 16 step.
// The order that leaves -- elements 0,4,1,5,2,6,3,7 -- is given to the other operand as well.  V's codes
// are transposed by the 4-bit transposing read: 16 lanes point at the rows of 16 keys, eight bytes each, and lane i receives column i.
constexpr int kQ4Wave = 64;       // keys per wave and step

// Two bf16 numbers 16 + code each for elements e and e + 4 of a word.  (The mask in a scalar register and the bias in a vector
// register: as literals they would take an instruction each.)
struct CodeBits { unsigned mask, bias; };
__device__ __forceinline__ CodeBits code_bits() {
  CodeBits b;
  asm("s_mov_b32 %0, 0x00780078" : "=s"(b.mask));
  asm("v_mov_b32 %0, 0x41804180" : "=v"(b.bias));
  return b;
}
__device__ __forceinline__ bf16x8 codes8(unsigned w, const CodeBits& b) {
  return __builtin_bit_cast(bf16x8, u32x4{((w << 3) & b.mask) | b.bias, ((w >> 1) & b.mask) | b.bias,
                                          ((w >> 5) & b.mask) | b.bias, ((w >> 9) & b.mask) | b.bias});
}

// A work-group's waves take the kv heads of one stretch of keys, 64 keys per wave and step.  The rows of a step -- the codes and
// the pairs of the work-group's heads, whole lines of memory -- go straight into LDS, all waves loading, while the step before it
// is worked on.  (Every wave loading the pieces of its own head instead asks the first-level cache for
// every line eight times over, and 131072 cached tokens of 8 heads took 44 us.)  A row's 16-byte
// pieces are permuted so that the transposing reads of 64 rows spread over the banks.
template <int D> constexpr int kQ4Places = D == 64 ? 18 : 36;      // 16-byte pieces of a key and step at most (times 64 keys: LDS)

// The steps of all sequences stand in a row, sequence after sequence, and are cut evenly among the work-groups: the lengths are
// known here and not on the host, and a ragged batch keeps every CU busy to the end.  A run may cover several sequences; the
// piece of sequence r that work-group i leaves has number i + r, which no other pair has (along the row one of the two grows).
// Work-group 0 leaves the first step of every sequence for the kernel that joins.
struct Q4Cut {      // total steps among at most `groups` work-groups: the first `more` of them take one step more than the others
  unsigned groups, each, more;
  __device__ __forceinline__ Q4Cut(unsigned total, unsigned most) {
    groups = total < most ? total : most;      // (every one that takes part has a step)
    each = groups > 0 ? total / groups : 0;
    more = total - each * groups;
  }
  __device__ __forceinline__ unsigned first(unsigned i) const { return i * each + (i < more ? i : more); }
  __device__ __forceinline__ unsigned owner(unsigned step) const {
    const unsigned wide = more * (each + 1);
    return step < wide ? step / (each + 1) : more + (step - wide) / each;
  }
};

struct Q4Run { int r, len; unsigned from, to, seq_first; };      // steps from .. to, beginning in sequence r
// own_len: the length of sequence threadIdx.x, asked for before.
template <int THREADS>
__device__ __forceinline__ bool q4_run(const Q4AttnArgs& a, int step_keys, int own_len, unsigned* sm, Q4Run& run) {
  constexpr int WAVES = THREADS / 64;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool notes = blockIdx.x == 0 && blockIdx.z == 0;
  const int chunks = (a.R + THREADS - 1) / THREADS;
  unsigned total = 0;
  // (batches of up to THREADS sequences: one look at the lengths; more: one for the total, one for the place)
  for (int pass = chunks > 1 ? 0 : 1; pass < 2; ++pass) {
    unsigned before = 0;
    for (int c = 0; c < chunks; ++c) {
      const int r = c * THREADS + tid;
      const int len = r < a.R ? imin(imax(c == 0 ? own_len : a.kv_len[r], 0), a.max_len) : 0;
      const unsigned n = (unsigned)(len + step_keys - 1) / (unsigned)step_keys;
      unsigned sum = n;
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const unsigned other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
      }
      if (lane == 63) sm[wave] = sum;
      __syncthreads();
      unsigned chunk = 0;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        if (w == wave) sum += chunk;
        chunk += sm[w];
      }
      if (pass == 1) {
        if (chunks == 1) total = chunk;
        const unsigned at = before + sum - n;
        const Q4Cut cut(total, gridDim.x);
        const unsigned from = blockIdx.x < cut.groups ? cut.first(blockIdx.x) : total;
        if (notes && r < a.R) a.seq_step[r] = at;
        if (notes && r == a.R - 1) a.seq_step[a.R] = before + sum;
        if (from >= at && from < at + n) {
          sm[WAVES] = (unsigned)r;
          sm[WAVES + 1] = at;
          sm[WAVES + 2] = (unsigned)len;
        }
      }
      before += chunk;
      __syncthreads();
    }
    if (pass == 0) total = before;
  }
  const Q4Cut cut(total, gridDim.x);
  if (blockIdx.x >= cut.groups) return false;
  run.from = cut.first(blockIdx.x);
  run.to = cut.first(blockIdx.x + 1);
  run.r = __builtin_amdgcn_readfirstlane(sm[WAVES]);
  run.seq_first = __builtin_amdgcn_readfirstlane(sm[WAVES + 1]);
  run.len = __builtin_amdgcn_readfirstlane(sm[WAVES + 2]);
  return true;
}

template <int D, bool MASS>
__global__ __launch_bounds__(64 * q4_waves(D), q4_dense(D)) void k_q4_attn(Q4AttnArgs a) {
  constexpr int W = q4_waves(D), THREADS = 64 * W;
  constexpr int NG = D / kQ4Group;          // groups per head row
  constexpr int HP = D / 32;                // 16-byte pieces of a head's codes
  constexpr int SWAP = HP - 1 < 3 ? HP - 1 : 3;
  constexpr int DT = D / 16;
  constexpr int PLACES = kQ4Places<D>;
  constexpr int LOADS = (PLACES + W - 1) / W;          // loads of a wave per step and cache
  // (two variables per buffer: see the attention of packed batches)
  __shared__ __align__(16) u32x4 k0s[64 * PLACES], k1s[64 * PLACES], v0s[64 * PLACES], v1s[64 * PLACES];
  __shared__ __align__(16) f32x2 spair[W][NG][kQ4Wave];      // (step, offset) of a wave's keys: K's times c, then V's
  __shared__ long long rows0[kQ4Wave * kQ4MaxWaveParts], rows1[kQ4Wave * kQ4MaxWaveParts];      // byte offsets of a step's keys
  static_assert(kQ4Wave * kQ4MaxWaveParts <= THREADS, "a thread per key of a step");
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, l16 = lane & 15, quarter = lane >> 4;
  const int qtiles = (a.Gq + 15) / 16;
  const int q16 = (int)(blockIdx.z % qtiles) * 16;   // first query head of the group that this work-group takes
  const int head0 = a.wave_parts > 1 ? 0 : (int)(blockIdx.z / qtiles) * W;
  const int heads = a.wave_parts > 1 ? a.Hkv : imin(W, a.Hkv - head0);
  const int hw = wave / a.wave_parts, wp = wave % a.wave_parts;
  const int head = head0 + hw;
  const bool works = hw < heads;
  const CodeBits bits = code_bits();
  const int step_keys = kQ4Wave * a.wave_parts;

  // ---- staging.  A row in LDS: the codes of the work-group's heads (permuted pieces), then their pairs.  Load i of this wave
  // writes 64 consecutive pieces; where its lane's piece comes from inside which row does not change from step to step, nor from
  // K's row to V's
  const int own_len = a.kv_len[imin(tid, a.R - 1)];
  const int code_places = heads * HP, places = code_places + (heads * NG * 4 + 15) / 16;
  const int loads = a.wave_parts * places;      // per cache
  const unsigned places_magic = 0xFFFFFFFFu / (unsigned)places;
  int from_row[LOADS], from_at[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    unsigned row, place;
    divmod_by((unsigned)((i * W + wave) * 64 + lane), (unsigned)places, places_magic, row, place);
    from_row[i] = (int)row;
    from_at[i] = (int)place < code_places ? head0 * (D / 2) + (int)(place ^ ((row >> 2) & SWAP)) * 16
                                     : (int)q4_code_bytes(a.Hkv, D) + head0 * NG * 4 + ((int)place - code_places) * 16;
  }

  // ---- this work-group's run of steps
  Q4Run run;
  if (!q4_run<THREADS>(a, step_keys, own_len, (unsigned*)rows1, run)) return;
  int r = run.r;

  u32x4 qf[NG][2];
  float qsum[NG];
  const bool live = works && q16 + l16 < a.Gq;
  // queries of sequence r: lane = query head q16 + l16, element order of the codes
  auto load_queries = [&]() __attribute__((always_inline)) {
    const char* src = a.q + (long long)r * a.q_stride_b + (long long)(imin(head, a.Hkv - 1) * a.Gq + imin(q16 + l16, a.Gq - 1)) * (D * 2);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      float sum = 0.0f;
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const u32x4 w = *(const u32x4*)(src + g * 128 + quarter * 32 + s * 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += bf16_lo(w[i]) + bf16_hi(w[i]);
        // words (e0,e1)(e2,e3)(e4,e5)(e6,e7) -> (e0,e4)(e1,e5)(e2,e6)(e3,e7)
        qf[g][s] = u32x4{(w.x & 0xffffu) | (w.z << 16), (w.x >> 16) | (w.z & 0xffff0000u),
                         (w.y & 0xffffu) | (w.w << 16), (w.y >> 16) | (w.w & 0xffff0000u)};
      }
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      qsum[g] = sum;
    }
  };

  f32x4 o[DT], ow[NG];                          // weighted codes; sums of the rounded weights * steps (every row of it the same)
  float m, l, ol[NG];                           // reference, sum of weights, sum of weights * offsets
  int len = 0, first = 0, last = 0;             // the sequence's length; its keys that this work-group takes

  auto stage = [&](const long long* rows, u32x4* sk, u32x4* sv) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int j = i * W + wave;
      if (j < loads) {
        const long long at = rows[from_row[i]] + from_at[i];
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(a.k + at),
                                         (__attribute__((address_space(3))) void*)(sk + j * 64), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(a.v + at),
                                         (__attribute__((address_space(3))) void*)(sv + j * 64), 16, 0, 0);
      }
    }
  };
  // byte offset of this thread's key of the step at k0 (keys past the end repeat the last one)
  auto row_offset = [&](int k0) __attribute__((always_inline)) -> long long {
    unsigned blk, at;
    divmod_by((unsigned)imin(k0 + tid, len - 1), (unsigned)a.kv_block, a.kv_magic, blk, at);
    return ((long long)a.block_table[(long long)r * a.table_stride + blk] * a.kv_block + at) * a.cache_stride;
  };

  // ---- one step: this wave's 64 keys from ks on, in LDS
  auto step = [&](int ks, const u32x4* sk, const u32x4* sv) __attribute__((always_inline)) {
    if (!works || ks >= last) return;
    const int row0 = wp * kQ4Wave;
    auto pair_of = [&](const u32x4* buf, int g) { return ((const unsigned*)(buf + (row0 + lane) * places + code_places))[hw * NG + g]; };
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const unsigned w = pair_of(sk, g);
      const float st = bf16_hi(w) * a.c;
      spair[wave][g][lane] = f32x2{st, fmaf(-16.0f, st, bf16_lo(w) * a.c)};
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // ---- logits in log2 units: x[t][j] of key ks + 16t + 4*quarter + j
    float x[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const int row = row0 + 16 * t + l16;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const u32x2 kc = ((const u32x2*)(sk + row * places + ((hw * HP + 2 * g + (quarter >> 1)) ^ ((row >> 2) & SWAP))))[quarter & 1];
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8(kc.x, bits), __builtin_bit_cast(bf16x8, qf[g][0]), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8(kc.y, bits), __builtin_bit_cast(bf16x8, qf[g][1]), acc, 0, 0, 0);
        const f32x4* pr = (const f32x4*)&spair[wave][g][16 * t + 4 * quarter];
        const f32x4 p01 = pr[0], p23 = pr[1];
        const float add = qsum[g];
        x[t][0] = fmaf(p01.x, acc[0], g == 0 ? p01.y * add : fmaf(p01.y, add, x[t][0]));
        x[t][1] = fmaf(p01.z, acc[1], g == 0 ? p01.w * add : fmaf(p01.w, add, x[t][1]));
        x[t][2] = fmaf(p23.x, acc[2], g == 0 ? p23.y * add : fmaf(p23.y, add, x[t][2]));
        x[t][3] = fmaf(p23.z, acc[3], g == 0 ? p23.w * add : fmaf(p23.w, add, x[t][3]));
      }
      __builtin_amdgcn_sched_barrier(0);      // (keeps the registers of one tile's codes from living beside the next's)
    }
    if (MASS && live) {
      float* dst = a.logits + ((long long)r * a.Hq + head * a.Gq + q16 + l16) * a.logit_stride + ks + 4 * quarter;
#pragma unroll
      for (int t = 0; t < 4; ++t) *(f32x4*)(dst + 16 * t) = f32x4{x[t][0], x[t][1], x[t][2], x[t][3]};
    }
    if (ks + kQ4Wave > last) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (ks + 16 * t + 4 * quarter + j >= len) x[t][j] = -INFINITY;
    }
    // V's offset stands for code 8, the middle: what a weight's rounding multiplies is then code - 8 (24 = 16 + 8 times the rounded
    // weights are taken back at the end), and not the lowest value or code + 16
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const unsigned w = pair_of(sv, g);
      spair[wave][g][lane] = f32x2{bf16_hi(w), fmaf(8.0f, bf16_hi(w), bf16_lo(w))};
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // ---- running softmax (the first key of a step is always there: no row without a maximum)
    float mx = x[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 4; j += 2) mx = fmaxf(fmaxf(mx, x[t][j]), x[t][j + 1]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    if (__any(mx > m)) {
      const float up = fmaxf(m, mx), f = exp2_of(m - up);
      m = up;
      l *= f;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        ol[g] *= f;
#pragma unroll
        for (int j = 0; j < 4; ++j) ow[g][j] *= f;
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[dt][j] *= f;
    }
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[t][j] = exp2_of(x[t][j] - m);
        l += x[t][j];
      }
    // ---- values.  Word 0 of a transposed read: keys 4*quarter + j of tiles 0 and 1, word 1: of tiles 2 and 3
    const bf16x8 ones = __builtin_bit_cast(bf16x8, u32x4{0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u});
    const int vrow = row0 + 16 * (l16 >> 2) + 4 * quarter + (l16 & 3);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      bf16x8 pw[2];
#pragma unroll
      for (int mm = 0; mm < 2; ++mm) {
        const f32x4* pa = (const f32x4*)&spair[wave][g][32 * mm + 4 * quarter];
        const f32x4* pb = (const f32x4*)&spair[wave][g][32 * mm + 16 + 4 * quarter];
        const f32x4 a01 = pa[0], a23 = pa[1], b01 = pb[0], b23 = pb[1];
        const float sa[4] = {a01.x, a01.z, a23.x, a23.z}, la[4] = {a01.y, a01.w, a23.y, a23.w};
        const float sb[4] = {b01.x, b01.z, b23.x, b23.z}, lb[4] = {b01.y, b01.w, b23.y, b23.w};
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float wa = x[2 * mm][j], wb = x[2 * mm + 1][j];
          w[j] = pack2(wa * sa[j], wb * sb[j]);
          ol[g] = fmaf(wa, la[j], fmaf(wb, lb[j], ol[g]));
        }
        pw[mm] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
        ow[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, pw[mm], ow[g], 0, 0, 0);
      }
#pragma unroll
      for (int dd = 0; dd < 4; ++dd) {
        const int dt = g * 4 + dd;
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) i32x2* lds2;
        const u32x4* at = sv + vrow * places + ((hw * HP + (dt >> 1)) ^ ((vrow >> 2) & SWAP));
        const i32x2 vt = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds2)((__attribute__((address_space(3))) char*)at + (dt & 1) * 8));
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8((unsigned)vt.x, bits), pw[0], o[dt], 0, 0, 0);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8((unsigned)vt.y, bits), pw[1], o[dt], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  // ---- the row offsets run two steps ahead, the rows one
  const bool looks = tid < step_keys;
  auto staged = [&]() __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    __syncthreads();
  };
  len = run.len;
  while (true) {
    const int seq_steps = (len + step_keys - 1) / step_keys;
    const int here = (int)(run.from - run.seq_first), n = imin((int)(run.to - run.from), seq_steps - here);
    const bool whole = n == seq_steps;        // the sequence is all here: the output is final
    first = here * step_keys;
    last = n == seq_steps - here ? len : first + n * step_keys;
    load_queries();
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) { ol[g] = 0.0f; ow[g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f}; }
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    long long at0 = 0, at1 = 0;
    if (looks) {
      at0 = row_offset(first);
      at1 = row_offset(imin(first + step_keys, last - 1));
    }
    __syncthreads();      // (rows1 held the run)
    if (looks) {
      rows0[tid] = at0;
      rows1[tid] = at1;
    }
    __syncthreads();
    stage(rows0, k0s, v0s);
    staged();
    for (int ks = first; ks < last; ks += 2 * step_keys) {
      long long ahead = 0;
      if (looks) ahead = row_offset(imin(ks + 2 * step_keys, last - 1));
      if (ks + step_keys < last) stage(rows1, k1s, v1s);
      step(ks + wp * kQ4Wave, k0s, v0s);
      if (looks) rows0[tid] = ahead;
      staged();
      if (ks + step_keys >= last) break;
      if (looks) ahead = row_offset(imin(ks + 3 * step_keys, last - 1));
      if (ks + 2 * step_keys < last) stage(rows0, k0s, v0s);
      step(ks + step_keys + wp * kQ4Wave, k1s, v1s);
      if (looks) rows1[tid] = ahead;
      staged();
    }

    // ---- o[dt][j]: element 16*dt + 4*quarter + j of query head q16 + l16
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      ol[g] += __shfl_xor(ol[g], 16);
      ol[g] += __shfl_xor(ol[g], 32);
      ol[g] = fmaf(-24.0f, ow[g][0], ol[g]);
    }
    const long long hq = head * a.Gq + q16 + l16;
    if (live && whole && a.wave_parts == 1) {
      const float inv = 1.0f / l;
      char* dst = a.out + (long long)r * a.out_stride_b + hq * (D * 2);
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const float b = ol[dt / 4];
        *(u32x2*)(dst + (dt * 16 + quarter * 4) * 2) =
            u32x2{pack2((o[dt][0] + b) * inv, (o[dt][1] + b) * inv), pack2((o[dt][2] + b) * inv, (o[dt][3] + b) * inv)};
      }
      const float lse2 = m + __log2f(l);
      if (quarter == 0 && a.lse != nullptr) a.lse[hq * a.lse_stride + r] = lse2 * 0.69314718055994530942f;
      if (quarter == 0 && MASS) a.lse2[(long long)r * a.Hq + hq] = lse2;
    } else if (live) {
      // (a wave without a key: reference -inf, sums 0)
      const long long at = (((long long)blockIdx.x + r) * a.wave_parts + wp) * a.Hq + hq;
#pragma unroll
      for (int dt = 0; dt < DT; ++dt) {
        const float b = ol[dt / 4];
        *(f32x4*)(a.o_part + at * D + dt * 16 + quarter * 4) = f32x4{o[dt][0] + b, o[dt][1] + b, o[dt][2] + b, o[dt][3] + b};
      }
      if (quarter == 0) {
        a.ml_part[2 * at] = m;
        a.ml_part[2 * at + 1] = l;
      }
    }
    run.from += n;
    if (run.from >= run.to) return;
    run.seq_first += seq_steps;
    do len = imin(a.kv_len[++r], a.max_len); while (len <= 0);      // (the run goes on: a sequence with keys follows)
  }
}

// Joins the pieces of one query head of one sequence: the work-group's waves take the pieces in turn, eight in flight each, and
// their sums are added in order.
template <int D>
__global__ __launch_bounds__(64 * kQ4JoinWaves) void k_q4_join(Q4AttnArgs a) {
  constexpr int PER = D / 64, FLY = 8;
  __shared__ float sacc[kQ4JoinWaves][D], sl[kQ4JoinWaves], sm[kQ4JoinWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
  const int r = blockIdx.y, hq = blockIdx.x;
  // steps p0 .. p1 of the row belong to this sequence, and the work-groups from i0 to i1 took them (see q4_run)
  const unsigned p0s = a.seq_step[r], p1s = a.seq_step[r + 1];
  const bool empty = p0s == p1s;
  const Q4Cut cut(a.seq_step[a.R], (unsigned)a.groups);
  const int i0 = empty ? 0 : (int)cut.owner(p0s), i1 = empty ? -1 : (int)cut.owner(p1s - 1);
  if (i0 == i1 && a.wave_parts == 1) return;      // the one that took it all has written the output
  const int live = (i1 - i0 + 1) * a.wave_parts;
  const long long at0 = ((long long)i0 + r) * a.wave_parts * a.Hq + hq;
  float m = -INFINITY;
  for (int p = threadIdx.x; p < live; p += blockDim.x) m = fmaxf(m, a.ml_part[2 * (at0 + (long long)p * a.Hq)]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  if (lane == 0) sm[wave] = m;
  __syncthreads();
  m = sm[0];
  for (int w = 1; w < waves; ++w) m = fmaxf(m, sm[w]);
  float l = 0.0f, acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.0f;
  for (int p0 = wave; p0 < live; p0 += waves * FLY) {
    float pm[FLY], pl[FLY], po[FLY][PER];
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const long long at = at0 + (long long)imin(p0 + waves * u, live - 1) * a.Hq;
      pm[u] = a.ml_part[2 * at];
      pl[u] = a.ml_part[2 * at + 1];
#pragma unroll
      for (int i = 0; i < PER; ++i) po[u][i] = a.o_part[at * D + i * 64 + lane];
    }
#pragma unroll
    for (int u = 0; u < FLY; ++u) {
      const float f = p0 + waves * u < live ? exp2_of(pm[u] - m) : 0.0f;
      l = fmaf(pl[u], f, l);
#pragma unroll
      for (int i = 0; i < PER; ++i) acc[i] = fmaf(po[u][i], f, acc[i]);
    }
  }
#pragma unroll
  for (int i = 0; i < PER; ++i) sacc[wave][i * 64 + lane] = acc[i];
  if (lane == 0) sl[wave] = l;
  __syncthreads();
  if (threadIdx.x >= D) return;
  float sum = 0.0f;
  l = 0.0f;
  for (int w = 0; w < waves; ++w) {
    l += sl[w];
    sum += sacc[w][threadIdx.x];
  }
  __bf16* dst = (__bf16*)(a.out + (long long)r * a.out_stride_b + (long long)hq * (D * 2));
  dst[threadIdx.x] = (__bf16)(empty ? 0.0f : sum * (1.0f / l));
  const float lse2 = empty ? -INFINITY : m + __log2f(l);
  if (threadIdx.x == 0 && a.lse != nullptr) a.lse[(long long)hq * a.lse_stride + r] = lse2 * 0.69314718055994530942f;
  if (threadIdx.x == 0 && a.lse2 != nullptr) a.lse2[(long long)r * a.Hq + hq] = lse2;
}

// Accumulated weight: the query heads' weights of a token added in order, their mean onto what it had.
__global__ __launch_bounds__(256) void k_q4_mass(Q4AttnArgs a) {
  const int r = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  if (i >= len) return;
  const float* x = a.logits + (long long)r * a.Hq * a.logit_stride + i;
  float sum = 0.0f;
#pragma unroll 8
  for (int h = 0; h < a.Hq; ++h) sum += exp2_of(x[h * a.logit_stride] - a.lse2[(long long)r * a.Hq + h]);
  const long long at = (long long)r * a.mass_stride + i;
  a.mass_out[at] = (a.mass_in != nullptr ? a.mass_in[at] : 0.0f) + sum / (float)a.Hq;
}

template <int D, bool MASS>
hipError_t launch_q4_pass(const Q4AttnArgs& a, hipStream_t s) {
  const dim3 grid(a.groups, 1, a.head_groups * ((a.Gq + 15) / 16)), block(64 * q4_waves(D));
  hipLaunchKernelGGL((k_q4_attn<D, MASS>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <int D>
hipError_t launch_q4_attn(const Q4AttnArgs& a, hipStream_t s) {
  hipError_t e = a.mass_out != nullptr ? launch_q4_pass<D, true>(a, s) : launch_q4_pass<D, false>(a, s);
  if (e != hipSuccess) return e;
  // (up to eight pieces per wave: one round of loads)
  const int waves = a.groups * a.wave_parts > 32 * a.R ? kQ4JoinWaves : 4;
  hipLaunchKernelGGL((k_q4_join<D>), dim3(a.Hq, a.R), dim3(64 * waves), 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.mass_out != nullptr && a.max_len > 0) {
    hipLaunchKernelGGL(k_q4_mass, dim3((a.max_len + 255) / 256, a.R), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

dim3 q4_copy_grid(const Q4CopyArgs& a) {
  const long long units = a.n * a.heads * (a.D / kQ4Group), each = kQ4Block;
  return dim3((unsigned)((units + each - 1) / each), 2);
}

}  // namespace

hipError_t launch_q4_store(const Q4CopyArgs& a, bool f32, hipStream_t s) {
  const dim3 grid = q4_copy_grid(a);
  if (f32) hipLaunchKernelGGL((k_q4_store<true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_q4_store<false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_q4_load(const Q4CopyArgs& a, bool f32, hipStream_t s) {
  const dim3 grid = q4_copy_grid(a);
  if (f32) hipLaunchKernelGGL((k_q4_load<true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_q4_load<false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_q4_attention(const Q4AttnArgs& a, hipStream_t s) {
  if (a.D == 64) return launch_q4_attn<64>(a, s);
  if (a.D == 128) return launch_q4_attn<128>(a, s);
  return launch_q4_attn<256>(a, s);
}

}  // namespace up
