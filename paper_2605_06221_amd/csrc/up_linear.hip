// Linear attention with a decay for each kv head (lam = exp(log_decay), at most 1):
//     S_t = lam S_{t-1} + k_t^T v_t,        out_t = scale q_t S_t      (S: D x D, float, carried by the sequence)
//
// k_linear_step: one token per sequence.  k_linear, k_linear_join: prompts and chunks, 32 tokens at a time on the matrix cores.
#include "up_attn.h"
#include "up_layers.h"

namespace up {

__device__ __forceinline__ float linear_load(const char* p, int i, bool f32) {
  return f32 ? ((const float*)p)[i] : __builtin_bit_cast(float, (unsigned)((const unsigned short*)p)[i] << 16);
}

// exp(log_decay * n) as a float and what it lacks, relative to it: a state is scaled once per step, and the error of one float would add
// up over the steps
__device__ __forceinline__ void linear_decay(float log_decay, int n, float& one, float& lacks) {
  const double x = exp((double)fminf(fmaxf(log_decay, -1e4f), 0.0f) * (double)n);
  one = (float)x;
  lacks = one > 1e-30f ? (float)((x - (double)one) / (double)one) : 0.0f;
}

__device__ __forceinline__ long long linear_slot(const int32_t* of, int r, long long num) {
  if (of == nullptr) return -1;
  const long long s = of[r];
  return s >= 0 && s < num ? s : -1;
}

// One token per sequence.  A work-group holds 32 columns of a head's state in registers, eight lanes by 32 groups of rows: every row's 128 bytes
// are read and written whole, and even a single sequence of few heads has work-groups for some tens of CUs.  Bound by the states' bytes
// (64 sequences of 32 heads of 128: 59 us, 4.6 TB/s, 91 % of a copy's rate; one sequence: a launch).
template <bool F32, int D>
__global__ __launch_bounds__(256) void k_linear_step(LinearArgs a) {
  constexpr int SLICES = D / 32, PER = D / 32, E = F32 ? 4 : 2;      // rows of the state per lane
  const int slice = blockIdx.x % SLICES, kvh = (blockIdx.x / SLICES) % a.Hkv, r = blockIdx.x / (SLICES * a.Hkv);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = slice * 32 + (lane & 7) * 4, row0 = (wave * 8 + (lane >> 3)) * PER;
  __shared__ f32x4 part[2][4][8];
  const long long from = linear_slot(a.state_in, r, a.num_states), to = linear_slot(a.state_out, r, a.num_states);
  const long long state_at = ((long long)kvh * D + row0) * D + col;
  const char* k = a.k + (long long)r * a.k_stride_b + (long long)kvh * D * E;
  const char* v = a.v + (long long)r * a.v_stride_b + (long long)kvh * D * E;
  f32x4 S[PER], v4;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    S[i] = f32x4{0, 0, 0, 0};
    if (from >= 0) S[i] = *(const f32x4*)(a.states + from * a.state_stride + state_at + i * D);
  }
  float one, lacks;
  linear_decay(a.log_decay[kvh], 1, one, lacks);
  const float rest = one * lacks;
#pragma unroll
  for (int i = 0; i < 4; ++i) v4[i] = linear_load(v, col + i, F32);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const float ki = linear_load(k, row0 + i, F32);
#pragma unroll
    for (int e = 0; e < 4; ++e) S[i][e] = fmaf(ki, v4[e], fmaf(S[i][e], one, S[i][e] * rest));
    if (to >= 0) *(f32x4*)(a.states + to * a.state_stride + state_at + i * D) = S[i];
  }
  for (int g = 0; g < a.Gq; ++g) {
    const int h = kvh * a.Gq + g;
    const char* q = a.q + (long long)r * a.q_stride_b + (long long)h * D * E;
    f32x4 o = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float qi = linear_load(q, row0 + i, F32);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = fmaf(qi, S[i][e], o[e]);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      for (int d = 8; d < 64; d <<= 1) o[e] += __shfl_xor(o[e], d);
    if (lane < 8) part[g & 1][wave][lane] = o;
    __syncthreads();      // (two buffers: the readers of this one are through before it is written again)
    if (tid < 8) {
      const f32x4 p0 = part[g & 1][0][tid], p1 = part[g & 1][1][tid], p2 = part[g & 1][2][tid], p3 = part[g & 1][3][tid];
      char* dst = a.out + (long long)r * a.out_stride_b + (long long)h * D * E;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = ((p0[e] + p1[e]) + (p2[e] + p3[e])) * a.scale;
        if (F32) ((float*)dst)[col + e] = y;
        else ((__bf16*)dst)[col + e] = (__bf16)y;
      }
    }
  }
}

// ---- chunks
//
// Chunks of 32 tokens: with i, j the tokens' places in the chunk and S the state before it,
//     out_i = scale (lam^(i+1) q_i S + sum_{j<=i} lam^(i-j) <q_i, k_j> v_j),       S <- lam^m S + sum_j k_j^T (lam^(m-1-j) v_j)
// (m tokens in the chunk).  A work-group walks over the chunks of one kv head, a wave holding 32 columns of the state in accumulators;
// all the wave's products have its columns as lanes or rows, so that waves share tiles of q, k and v in LDS and nothing else:
//     P^T = K Q^T,    O^T = S^T Q^T (scaled) + V^T P^T,    S += K^T V'
// P^T and S leave the matrix cores in the layout that an operand of the next product has: the contraction takes keys (elements of a key)
// in the order in which the lanes hold them.  K^T and V^T come out of row-major LDS through the transposing read.
//
// Products of bf16 are exact and summed in float.  What is scaled first is no bf16 any more: P and S enter the products for the outputs
// in two parts of bf16 (16 bits), V' the one for the state in three (24 bits: what the state adds up over a long sequence stays float).
//
// Long sequences are cut into pieces of `piece` tokens: one launch leaves what every piece adds to the state, a second
// adds these up in order, and the third walks over the pieces from the states that they begin with.  Keys and values are then read twice.
//
// What bounds it: at one query head per kv head the bytes with the SIMDs full as well (a prompt of 32768, 32 heads of 128, 407 to 440 us; its launches at
// their fastest 126, 537 MB, and 259, 1.07 GB, both at 4.2 TB/s, and 19 for the join, with medians of 153, 311 and 21 in a profiled run; in the third
// the matrix cores are busy in 41 % of the cycles, the vector pipe in 65 %: most of that is taking the state apart).  With several query heads per kv head a step's own latency, about 2 us
// from tiles to outputs, with few waves to fill it (40/8 heads of 64: matrix cores busy in 16 % of the cycles, vector pipe in 23 %): 32/8 heads 231 to 255 us.
// What it took (the same prompt): token after token 40.8 ms; chunks through registers into LDS, states scaled every chunk 490 us; two buffers and
// one barrier a chunk 469; straight into LDS, scaled when needed, three work-groups a CU instead of two 408.  The state's parts kept
// over the query heads, 16-byte stores and no wait for them: 32/8 heads 292 -> 259 us; eight pieces under way in the join: 8000 tokens of 8/8 heads of 64 40 -> 30.
constexpr int kLinearChunk = 32;
constexpr float kLinearUnit = 0x1p24f;      // what the state is divided by when it was last scaled (below)
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ unsigned linear_pack(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}
__device__ __forceinline__ float low_half(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float high_half(unsigned w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
// Eight floats in one part of bf16, and what is left of them (exact).
__device__ __forceinline__ u32x4 linear_part(float* x) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned part = linear_pack(x[2 * i], x[2 * i + 1]);
    x[2 * i] -= low_half(part);
    x[2 * i + 1] -= high_half(part);
    w[i] = part;
  }
  return w;
}
__device__ __forceinline__ u32x4 linear_last_part(const float* x) {
  return u32x4{linear_pack(x[0], x[1]), linear_pack(x[2], x[3]), linear_pack(x[4], x[5]), linear_pack(x[6], x[7])};
}
__device__ __forceinline__ f32x16 linear_mfma(const u32x4& a, const u32x4& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 linear_mfma(float a, float b, const f32x16& c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

// Tiles in LDS: 32 rows of PPR pieces of 16 bytes, the pieces of a row permuted so that both 16 rows' same piece and 4 rows' neighbouring
// pieces lie in different banks.
template <int PPR>
__device__ __forceinline__ int linear_swap(int row) { return PPR == 8 ? ((row & 2) << 1) | ((row >> 2) & 3) : ((row & 3) << 2) | ((row >> 2) & 3); }

template <bool F32, int D>
struct LinearTile {
  static constexpr int WAVES = D / 32, THREADS = 64 * WAVES, SRCB = D * (F32 ? 4 : 2), PPR = SRCB / 16;
  static constexpr int LOADS = kLinearChunk * PPR / THREADS;      // pieces per thread and tile
  static constexpr int KT = D / 32;                               // tiles of 32 elements along a key
  static constexpr int DENSE = D == 256 || F32 ? 2 : 3;           // waves per SIMD that the registers are held to
};

// place of a piece of the work: sequence r from its token t0 on, at most `piece` tokens
struct LinearPiece {
  int r, index, t0, tokens, length;      // t0: in the sequence; length: the sequence's
};
__device__ __forceinline__ bool linear_locate(const LinearArgs& a, int slot, LinearPiece& w) {
  w.r = locate_slot(a.cu, a.R, a.piece, slot);
  w.index = slot - slot_base(a.cu[w.r], w.r, a.piece);
  w.length = a.cu[w.r + 1] - a.cu[w.r];
  w.t0 = w.index * a.piece;
  w.tokens = imin(a.piece, w.length - w.t0);
  return w.tokens > 0 || w.index == 0;      // (a sequence without tokens hands its state on)
}
// what the piece adds (and later the state it begins with), in the workspace: sequences that are cut are longer than a piece, so they own
// floor(2 cu / piece) .. and as many as they have pieces
__device__ __forceinline__ float* linear_add(const LinearArgs& a, const LinearPiece& w, int D) {
  return a.adds + (2ll * a.cu[w.r] / a.piece + w.index) * a.Hkv * D * D;
}

// exp2(x * n), -120 <= x * n <= 0, to a float's rounding: a float's product would leave |x n| 2^-24 of error
__device__ __forceinline__ float linear_power(double x, int n) {
  const double y = x * (double)n, whole = rint(y);
  return ldexpf(__builtin_amdgcn_exp2f((float)(y - whole)), (int)whole);
}

template <bool F32, int D, bool OUT, bool HOLD>
__global__ __launch_bounds__(64 * (D / 32), (HOLD && D == 128 ? 2 : LinearTile<F32, D>::DENSE)) void k_linear(LinearArgs a) {
  typedef LinearTile<F32, D> T;
  constexpr int TILE = kLinearChunk * T::PPR;
  // keys, values and queries of a step, and of the next one.  (Two variables, not one array: the compiler then knows that a load into one and
  // reads of the other do not meet, and does not wait for the load before them.)
  __shared__ __align__(16) u32x4 tiles0[(OUT ? 3 : 2) * TILE], tiles1[(OUT ? 3 : 2) * TILE];
  __shared__ __align__(16) float value_weight[kLinearChunk];
  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = blockIdx.x % a.Hkv;
  LinearPiece w;
  if (!linear_locate(a, blockIdx.x / a.Hkv, w)) return;
  const bool cut = w.length > a.piece;
  const long long to = linear_slot(a.state_out, w.r, a.num_states);
  if (!OUT && !cut) return;
  if (!OUT && w.t0 + w.tokens == w.length && to < 0) return;      // (nobody asks for what the last piece adds)
  const long long first = (long long)a.cu[w.r] + w.t0;
  const double ld = (double)fminf(fmaxf(a.log_decay[kvh], -1e4f), 0.0f) * 1.4426950408889634074;
  const float ldf = (float)ld;

  // ---- the state: element e of S[kt] is row 32 kt + 8 (e / 4) + 4 half + e % 4, column 32 wave + l32
  const long long state_at = (long long)kvh * D * D + 4 * half * D + 32 * wave + l32;
  f32x16 S[T::KT];
  const float* from = nullptr;
  if (OUT && cut) from = linear_add(a, w, D);
  if (OUT && !cut) {
    const long long slot = linear_slot(a.state_in, w.r, a.num_states);
    if (slot >= 0) from = a.states + slot * a.state_stride;
  }
#pragma unroll
  for (int kt = 0; kt < T::KT; ++kt) {
#pragma unroll
    for (int e = 0; e < 16; ++e) S[kt][e] = 0.0f;
    if (from != nullptr) {
#pragma unroll
      for (int e = 0; e < 16; ++e) S[kt][e] = from[state_at + (32 * kt + 8 * (e >> 2) + (e & 3)) * D];
    }
    __builtin_amdgcn_sched_barrier(0);      // (a tile's addresses at a time)
  }

  // ---- weights: of the logits (token l32 against token 8 (e / 4) + 4 half + e % 4), of the state's product, of the values
  auto key_of = [&](int e) { return 8 * (e >> 2) + 4 * half + (e & 3); };
  float wp[OUT ? 16 : 1];
  if (OUT) {
#pragma unroll
    for (int e = 0; e < 16; ++e) wp[e] = key_of(e) <= l32 ? a.scale * __builtin_amdgcn_exp2f(ldf * (float)(l32 - key_of(e))) : 0.0f;
  }
  const float wo = a.scale * __builtin_amdgcn_exp2f(ldf * (float)(l32 + 1));
  auto weigh = [&](int m) {      // (tokens past the chunk's m weigh nothing)
    if (tid < kLinearChunk) value_weight[tid] = tid < m ? __builtin_amdgcn_exp2f(ldf * (float)(m - 1 - tid)) : 0.0f;
  };
  // The state stands in registers as S / (2^24 f), f = lam^(tokens since they were last scaled): it is scaled when f has passed 2^-24, not with
  // every chunk.  (The power of two changes no rounding: with it what stands there is never larger than the state itself, and a state
  // near the end of float's range does not leave it.  At the other end, below 2^-80, its low bits are lost.)
  int since = 0;
  float f = 1.0f;

  // ---- staging, straight from memory into LDS: a wave's load writes 64 consecutive places, WROWS rows; the permutation of a row's
  // pieces is in the address that the lane reads
  constexpr int WROWS = 64 / T::PPR, ROWSTEP = T::THREADS / T::PPR;
  unsigned koff[T::LOADS], voff[T::LOADS], qoff[OUT ? T::LOADS : 1];
  auto aim = [&](int rows) {      // rows past the end repeat the last one
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) {
      const int row = i * ROWSTEP + wave * WROWS + lane / T::PPR, piece = (lane % T::PPR) ^ linear_swap<T::PPR>(row), at = imin(row, rows - 1);
      koff[i] = (unsigned)at * (unsigned)a.k_stride_b + piece * 16;
      voff[i] = (unsigned)at * (unsigned)a.v_stride_b + piece * 16;
      if (OUT) qoff[i] = (unsigned)at * (unsigned)a.q_stride_b + piece * 16;
    }
  };
  const char* kbase = a.k + (long long)kvh * T::SRCB;
  const char* vbase = a.v + (long long)kvh * T::SRCB;
  const char* qbase = a.q + (long long)kvh * a.Gq * T::SRCB;
  auto stage = [&](int c0, int g, u32x4* tiles) __attribute__((always_inline)) {
    if (w.tokens - c0 < kLinearChunk) aim(w.tokens - c0);
    const char* k = kbase + (first + c0) * a.k_stride_b;
    const char* v = vbase + (first + c0) * a.v_stride_b;
    const char* q = qbase + (first + c0) * a.q_stride_b + g * T::SRCB;
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) {
      u32x4* to_row = tiles + (i * ROWSTEP + wave * WROWS) * T::PPR;
      load_to_lds(k + koff[i], to_row);
      load_to_lds(v + voff[i], to_row + TILE);
      if (OUT) load_to_lds(q + qoff[i], to_row + 2 * TILE);
    }
  };
  // Operands out of LDS.  row_part: the 16-byte piece `piece` + half of row l32 (piece even).  column_part: column 32 kt + l32 of the tile's rows 16 st + {4 half .. +3, 8 + 4 half .. +3}.
  // The place of a piece is that of piece 0 with the piece's bits turned over: one address a lane and an exclusive or each.
  unsigned row_at = l32 * T::SRCB + (linear_swap<T::PPR>(l32) ^ half) * 16;
  const int trow = 4 * half + ((lane >> 2) & 3), tpiece = ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1);
  unsigned col_at = F32 ? 4 * half * T::SRCB + (((l32 >> 2) ^ half) * 16) + (l32 & 3) * 4
                        : trow * T::SRCB + ((tpiece ^ linear_swap<T::PPR>(trow)) * 16) + (lane & 1) * 8;
  auto row_part = [&](const u32x4* tile, int piece) __attribute__((always_inline)) {
    return *(const u32x4*)((const char*)tile + (row_at ^ (piece * 16)));
  };
  // bf16 elements 8 half .. +7 of 16 -> 4 half .. +3 and 8 + 4 half .. +3, the order in which the lanes hold rows of the state
  auto state_order = [&](const u32x4& x) __attribute__((always_inline)) {
    const auto r0 = __builtin_amdgcn_permlane32_swap(x.x, x.z, false, false), r1 = __builtin_amdgcn_permlane32_swap(x.y, x.w, false, false);
    return u32x4{r0[0], r1[0], r0[1], r1[1]};
  };
  auto column_part = [&](const u32x4* tile, int kt, int st) __attribute__((always_inline)) {
    typedef __attribute__((address_space(3))) s16x4* lds4;
    auto at = [&](unsigned flip, int row) { return (lds4)(__attribute__((address_space(3))) char*)((const char*)tile + (col_at ^ (kt * 64) ^ flip) + row * T::SRCB); };
    const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(0, 16 * st)));
    const u32x2 y = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(32, 16 * st + 8)));      // (8 rows on, a swap's bit 1 is the other)
    return u32x4{x.x, x.y, y.x, y.y};
  };
  auto column_float = [&](const u32x4* tile, int kt, int e) __attribute__((always_inline)) {      // column 32 kt + l32 of row key_of(e)
    const int swap = ((e & 3) << 2) | ((2 * (e >> 2)) & 3);
    return *(const float*)((const char*)tile + (col_at ^ (kt * 128) ^ (swap * 16)) + (8 * (e >> 2) + (e & 3)) * T::SRCB);
  };

  // The state in two parts of bf16: taken apart for every head, or (HOLD: several query heads share the state) once a chunk and kept.
  u32x4 s1[HOLD ? T::KT : 1][2], s2[HOLD ? T::KT : 1][2];
  auto take_apart = [&](int kt, int st, u32x4& p1, u32x4& p2) __attribute__((always_inline)) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = S[kt][8 * st + i];
    p1 = linear_part(x);
    p2 = linear_last_part(x);
  };
  // one head's outputs for the chunk
  auto outputs = [&](int c0, int g, int m, const u32x4* sk, const u32x4* sv, const u32x4* sq) __attribute__((always_inline)) {
    f32x16 P, O;
#pragma unroll
    for (int e = 0; e < 16; ++e) P[e] = O[e] = 0.0f;
    constexpr bool AHEAD = !F32 && D == 128 && HOLD;
    u32x4 qs[2][2], ks[2][2];
#pragma unroll
    for (int kt = 0; kt < T::KT; ++kt) {
      if constexpr (F32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const u32x4 q4 = row_part(sq, 8 * kt + 2 * j), k4 = row_part(sk, 8 * kt + 2 * j);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float qf = __builtin_bit_cast(float, (unsigned)q4[i]), kf = __builtin_bit_cast(float, (unsigned)k4[i]);
            P = linear_mfma(kf, qf, P);
            O = linear_mfma(S[kt][4 * j + i], qf, O);
          }
        }
      } else {
        if (kt == 0 || !AHEAD) {
#pragma unroll
          for (int st = 0; st < 2; ++st) { qs[kt & 1][st] = row_part(sq, 4 * kt + 2 * st); ks[kt & 1][st] = row_part(sk, 4 * kt + 2 * st); }
        }
        if (AHEAD && kt + 1 < T::KT) {
#pragma unroll
          for (int st = 0; st < 2; ++st) { qs[(kt + 1) & 1][st] = row_part(sq, 4 * (kt + 1) + 2 * st); ks[(kt + 1) & 1][st] = row_part(sk, 4 * (kt + 1) + 2 * st); }
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
          const u32x4 q8 = qs[kt & 1][st], k8 = ks[kt & 1][st];
          P = linear_mfma(k8, q8, P);
          const int at = HOLD ? kt : 0;
          if (!HOLD) take_apart(kt, st, s1[0][st], s2[0][st]);
          const u32x4 q = state_order(q8);
          O = linear_mfma(s1[at][st], q, O);
          O = linear_mfma(s2[at][st], q, O);
        }
      }
      __builtin_amdgcn_sched_barrier(0);      // (the operands of one step at a time: all of them at once push accumulators into scratch)
    }
    const float wof = wo * (f * kLinearUnit);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      P[e] *= wp[e];
      O[e] *= wof;
    }
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 16; ++e) O = linear_mfma(column_float(sv, wave, e), P[e], O);
    } else {
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const u32x4 v8 = column_part(sv, wave, st);
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = P[8 * st + i];
        const u32x4 p1 = linear_part(x), p2 = linear_last_part(x);
        O = linear_mfma(v8, p1, O);
        O = linear_mfma(v8, p2, O);
      }
    }
    // Element e of O: token l32, column 32 wave + 8 (e / 4) + 4 half + e % 4.  Through a buffer that ends with the chunk's m rows, so that
    // a wave always issues all its stores (below).
    char* rows = a.out + (first + c0) * a.out_stride_b + (long long)(kvh * a.Gq + g) * T::SRCB;
    const auto buffer = __builtin_amdgcn_make_buffer_rsrc(rows, 0, (int)((unsigned)(m - 1) * (unsigned)a.out_stride_b + T::SRCB), 0x00027000);
    const unsigned at = (unsigned)l32 * (unsigned)a.out_stride_b + wave * 32 * (F32 ? 4 : 2) + half * 16;
    if constexpr (F32) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 x = {O[4 * j], O[4 * j + 1], O[4 * j + 2], O[4 * j + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, x), buffer, at + j * 32, 0, 0);
      }
    } else {      // (two quarters of 16 columns change lane halves: 16 bytes a lane)
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const auto r0 = __builtin_amdgcn_permlane32_swap(linear_pack(O[4 * j], O[4 * j + 1]), linear_pack(O[4 * j + 4], O[4 * j + 5]), false, false);
        const auto r1 = __builtin_amdgcn_permlane32_swap(linear_pack(O[4 * j + 2], O[4 * j + 3]), linear_pack(O[4 * j + 6], O[4 * j + 7]), false, false);
        __builtin_amdgcn_raw_buffer_store_b128(u32x4{r0[0], r1[0], r0[1], r1[1]}, buffer, at + j * 16, 0, 0);
      }
    }
  };
  // the state goes past the chunk: S += K^T V'.  In three parts where it is stored, in two where it only makes outputs.
  auto advance = [&](int m, const u32x4* sk, const u32x4* sv) __attribute__((always_inline)) {
    since += m;
    f = ldf * (float)since > -120.0f ? linear_power(ld, since) : 0.0f;      // (past 2^-120 nothing of it is left beside new tokens)
    f = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, f)));      // (the same for the whole wave: a branch)
    if (f < 0x1p-24f) {
#pragma unroll
      for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) S[kt][e] *= f;
      since = 0;
      f = 1.0f;
    }
    const float inv = (1.0f / kLinearUnit) / f;
    if constexpr (F32) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float x = column_float(sv, wave, e) * (value_weight[key_of(e)] * inv);
#pragma unroll
        for (int kt = 0; kt < T::KT; ++kt) S[kt] = linear_mfma(column_float(sk, kt, e), x, S[kt]);
      }
    } else {
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        const u32x4 v8 = column_part(sv, wave, st);
        float x[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const f32x4 wv = *(const f32x4*)&value_weight[16 * st + 8 * i + 4 * half];
          x[4 * i] = low_half(v8[2 * i]) * (wv[0] * inv);
          x[4 * i + 1] = high_half(v8[2 * i]) * (wv[1] * inv);
          x[4 * i + 2] = low_half(v8[2 * i + 1]) * (wv[2] * inv);
          x[4 * i + 3] = high_half(v8[2 * i + 1]) * (wv[3] * inv);
        }
        const u32x4 v1 = linear_part(x), v2 = linear_part(x);
#pragma unroll
        for (int kt = 0; kt < T::KT; ++kt) {
          const u32x4 k8 = column_part(sk, kt, st);
          S[kt] = linear_mfma(k8, v1, S[kt]);
          S[kt] = linear_mfma(k8, v2, S[kt]);
          if (!OUT) S[kt] = linear_mfma(k8, linear_last_part(x), S[kt]);
        }
        if (OUT && !cut) {      // (a pass of its own, in place)
          const u32x4 v3 = linear_last_part(x);
#pragma unroll
          for (int kt = 0; kt < T::KT; ++kt) S[kt] = linear_mfma(column_part(sk, kt, st), v3, S[kt]);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  // ---- steps: a chunk and a query head each; the next one's tiles are loaded while one is worked on
  if (w.tokens > 0) {
    aim(imin(kLinearChunk, w.tokens));
    weigh(imin(kLinearChunk, w.tokens));
    int c0 = 0, g = 0;
    auto step = [&](u32x4* here, u32x4* next) __attribute__((always_inline)) {      // false: the last one
      const bool last_head = !OUT || g == a.Gq - 1;
      const int m = imin(kLinearChunk, w.tokens - c0), c1 = last_head ? c0 + kLinearChunk : c0, g1 = last_head ? 0 : g + 1;
      const bool more = c1 < w.tokens;
      if (more) stage(c1, g1, next);
      // (made anew in every round: kept over the loop, addresses and the state's parts would push accumulators into scratch)
      asm volatile("" : "+v"(row_at), "+v"(col_at));
      if constexpr (HOLD) {
        if (g == 0) {
#pragma unroll
          for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
            for (int st = 0; st < 2; ++st) take_apart(kt, st, s1[kt][st], s2[kt][st]);
        }
      } else {
#pragma unroll
        for (int kt = 0; kt < T::KT; ++kt) asm volatile("" : "+v"(S[kt]));
      }
      if (OUT) outputs(c0, g, m, here, here + TILE, here + (OUT ? 2 * TILE : 0));
      if (last_head) advance(m, here, here + TILE);
      // The next tiles are in LDS and everyone is done with these.  Vector memory completes in order, and the step has issued its stores
      // since it asked for the tiles: these may be under way, which __syncthreads would wait for.
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(!OUT ? 0x0070 : F32 ? 0x0074 : 0x0072);      // vmcnt(0), (4), (2); lgkmcnt(0)
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
      if (last_head && more && w.tokens - c1 < kLinearChunk) {      // the last chunk is short
        weigh(w.tokens - c1);
        __syncthreads();
      }
      c0 = c1;
      g = g1;
      return more;
    };
    stage(0, 0, tiles0);
    __builtin_amdgcn_s_waitcnt(0x0f70);
    if (OUT) {      // (here, where the loads are waited for anyway)
#pragma unroll
      for (int kt = 0; kt < T::KT; ++kt)
#pragma unroll
        for (int e = 0; e < 16; ++e) S[kt][e] *= 1.0f / kLinearUnit;
    }
    __syncthreads();
    bool more;      // (one way out: a second one costs a second state in registers)
    do {
      more = step(tiles0, tiles1);
      if (more) more = step(tiles1, tiles0);
    } while (more);
  }
  float* dst = !OUT ? linear_add(a, w, D) : !cut && to >= 0 ? a.states + to * a.state_stride : nullptr;
  if (dst != nullptr) {
    const float unit = w.tokens > 0 ? f * kLinearUnit : 1.0f;
#pragma unroll
    for (int kt = 0; kt < T::KT; ++kt) {
#pragma unroll
      for (int e = 0; e < 16; ++e) dst[state_at + (32 * kt + 8 * (e >> 2) + (e & 3)) * D] = S[kt][e] * unit;
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// The states that the pieces of cut sequences begin with, from what every piece adds, in order; and the state afterwards.
template <int D>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs a) {
  constexpr int PARTS = D * D / 1024;
  const int part = blockIdx.x % PARTS, kvh = (blockIdx.x / PARTS) % a.Hkv;
  LinearPiece w;
  w.r = blockIdx.x / (PARTS * a.Hkv);
  w.length = a.cu[w.r + 1] - a.cu[w.r];
  w.index = 0;
  if (w.length <= a.piece) return;
  const long long at = (long long)kvh * D * D + part * 1024 + threadIdx.x * 4, step = (long long)a.Hkv * D * D;
  const long long from = linear_slot(a.state_in, w.r, a.num_states), to = linear_slot(a.state_out, w.r, a.num_states);
  f32x4 S = {0, 0, 0, 0};
  if (from >= 0) S = *(const f32x4*)(a.states + from * a.state_stride + at);
  float* add = linear_add(a, w, D) + at;
  float one, lacks;
  linear_decay(a.log_decay[kvh], a.piece, one, lacks);
  // (eight pieces' sums are under way together; the last piece's is added below, if anybody asks)
  const int before_last = (w.length - 1) / a.piece, left = w.length - before_last * a.piece;
  for (int i = 0; i < before_last; i += 8) {
    f32x4 x[8];
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i + u < before_last) x[u] = *(const f32x4*)(add + u * step);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (i + u >= before_last) break;
      *(f32x4*)add = S;
      add += step;
#pragma unroll
      for (int e = 0; e < 4; ++e) S[e] = fmaf(S[e], one, fmaf(S[e], one * lacks, x[u][e]));
    }
  }
  if (to >= 0) {
    const f32x4 x = *(const f32x4*)add;
    linear_decay(a.log_decay[kvh], left, one, lacks);
    f32x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = fmaf(S[e], one, fmaf(S[e], one * lacks, x[e]));
    *(f32x4*)(a.states + to * a.state_stride + at) = y;
  }
  *(f32x4*)add = S;
}

template <bool F32, int D>
static hipError_t launch_linear_form(const LinearArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)a.slots * a.Hkv), block(64 * (D / 32));
  if (a.adds != nullptr) {
    hipLaunchKernelGGL((k_linear<F32, D, false, false>), grid, block, 0, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((k_linear_join<D>), dim3((unsigned)a.R * a.Hkv * (D * D / 1024)), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  constexpr bool can_hold = !F32 && D <= 128;
  if (can_hold && a.Gq > 1) hipLaunchKernelGGL((k_linear<F32, D, true, can_hold>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_linear<F32, D, true, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

hipError_t launch_linear(const LinearArgs& a, bool f32, int D, hipStream_t s) {
  if (f32) return D == 64 ? launch_linear_form<true, 64>(a, s) : launch_linear_form<true, 128>(a, s);
  return D == 64 ? launch_linear_form<false, 64>(a, s) : D == 128 ? launch_linear_form<false, 128>(a, s) : launch_linear_form<false, 256>(a, s);
}

template <bool F32, int D>
static hipError_t launch_linear_step_form(const LinearArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_linear_step<F32, D>), dim3((unsigned)a.R * a.Hkv * (D / 32)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_linear_step(const LinearArgs& a, bool f32, int D, hipStream_t s) {
  if (f32) return D == 64 ? launch_linear_step_form<true, 64>(a, s) : launch_linear_step_form<true, 128>(a, s);
  return D == 64 ? launch_linear_step_form<false, 64>(a, s) : D == 128 ? launch_linear_step_form<false, 128>(a, s)
                                                                         : launch_linear_step_form<false, 256>(a, s);
}

}  // namespace up
