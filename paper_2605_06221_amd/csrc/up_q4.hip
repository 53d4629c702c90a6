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

// bits of the largest bf16 not above x, in the upper half of the word
__device__ __forceinline__ unsigned bf16_below(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x);
  return (b >> 31 ? b + 0xffffu : b) & 0xffff0000u;
}
// bits of the smallest bf16 not below x >= 0
__device__ __forceinline__ unsigned bf16_above(double x) {
  unsigned b = __builtin_bit_cast(unsigned, (float)x) & 0xffff0000u;
  if ((double)__builtin_bit_cast(float, b) < x) b += 0x10000u;
  return b;
}

// Eight lanes hold the 64 elements of a group, eight each.  A work-group takes kQ4Rows rows of keys and
// of values; its units are (row, keys or values, group), eight lanes per unit, so that a wave
// reads 1 KB of consecutive row bytes (bf16).
constexpr int kQ4Rows = 2;
struct Q4Unit { int t, kv, g; bool live; };
__device__ __forceinline__ Q4Unit q4_unit(const Q4CopyArgs& a, int unit, int groups, unsigned magic) {
  unsigned row, rest;
  divmod_by((unsigned)unit, 2u * groups, magic, row, rest);
  Q4Unit u;
  u.kv = (int)rest >= groups;
  u.g = (int)rest - u.kv * groups;
  const long long t = (long long)blockIdx.x * kQ4Rows + row;
  const long long n = a.count_dev != nullptr && a.count_dev[0] < a.n ? a.count_dev[0] : a.n;
  u.live = (int)row < kQ4Rows && t < n && a.cache[u.kv] != nullptr;
  u.t = (int)t;
  return u;
}

template <bool F32>
__global__ __launch_bounds__(256) void k_q4_store(Q4CopyArgs a) {
  const int groups = a.heads * (a.D / kQ4Group), sub = threadIdx.x & 7;
  const unsigned magic = 0xFFFFFFFFu / (2u * groups);
  const long long codes = q4_code_bytes(a.heads, a.D);
  for (int unit = threadIdx.x >> 3; unit < kQ4Rows * 2 * groups; unit += 32) {
    const Q4Unit u = q4_unit(a, unit, groups, magic);
    if (!u.live) continue;
    const int64_t slot = a.slots[u.t];
    if (slot < 0 || slot >= a.num_slots) continue;
    const char* src = a.rows_in[u.kv] + (long long)u.t * a.row_stride_b[u.kv] + (long long)(u.g * 8 + sub) * (F32 ? 32 : 16);
    float x[8];
    if (F32) {
      const f32x4 lo4 = ((const f32x4*)src)[0], hi4 = ((const f32x4*)src)[1];
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[i] = lo4[i]; x[4 + i] = hi4[i]; }
    } else {
      const u32x4 w = *(const u32x4*)src;
#pragma unroll
      for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(w[i]); x[2 * i + 1] = bf16_hi(w[i]); }
    }
    float mn = x[0], mx = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) { mn = fminf(mn, x[i]); mx = fmaxf(mx, x[i]); }
    mn = fminf(mn, lane_dpp<0xB1>(mn)); mx = fmaxf(mx, lane_dpp<0xB1>(mx));
    mn = fminf(mn, lane_dpp<0x4E>(mn)); mx = fmaxf(mx, lane_dpp<0x4E>(mx));
    mn = fminf(mn, lane_dpp<0x141>(mn)); mx = fmaxf(mx, lane_dpp<0x141>(mx));
    const unsigned lo_bits = bf16_below(mn);
    const float lo = __builtin_bit_cast(float, lo_bits);
    const unsigned step_bits = bf16_above(((double)mx - (double)lo) / 15.0);
    const float step = __builtin_bit_cast(float, step_bits);
    // The quotient in float is off by less than 2^-20 here; a code is decided in double where that could
    // matter (next to a half), and for steps whose reciprocal or range leaves the float range.
    const bool wide = !(step > 1e-30f && step < 1e30f);
    const float inv = 1.0f / step;
    unsigned packed = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float c = (x[i] - lo) * inv;
      const float off = c - floorf(c) - 0.5f;
      if (wide || fabsf(off) < 1e-3f) c = step > 0.0f ? (float)rint(((double)x[i] - (double)lo) / (double)step) : 0.0f;
      else c = rintf(c);
      const unsigned code = (unsigned)fminf(fmaxf(c, 0.0f), 15.0f);
      packed |= code << (4 * i);
    }
    char* dst = a.cache[u.kv] + (long long)slot * a.cache_stride;
    *(unsigned*)(dst + u.g * 32 + sub * 4) = packed;
    if (sub == 0) *(unsigned*)(dst + codes + (long long)u.g * 4) = (lo_bits >> 16) | step_bits;
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void k_q4_load(Q4CopyArgs a) {
  const int groups = a.heads * (a.D / kQ4Group), sub = threadIdx.x & 7;
  const unsigned magic = 0xFFFFFFFFu / (2u * groups);
  const long long codes = q4_code_bytes(a.heads, a.D);
  for (int unit = threadIdx.x >> 3; unit < kQ4Rows * 2 * groups; unit += 32) {
    const Q4Unit u = q4_unit(a, unit, groups, magic);
    if (!u.live) continue;
    const int64_t slot = a.slots[u.t];
    if (slot < 0 || slot >= a.num_slots) continue;
    const char* src = a.cache[u.kv] + (long long)slot * a.cache_stride;
    const unsigned packed = *(const unsigned*)(src + u.g * 32 + sub * 4);
    const unsigned pair = *(const unsigned*)(src + codes + (long long)u.g * 4);
    const float lo = bf16_lo(pair), step = bf16_hi(pair);
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = fmaf((float)((packed >> (4 * i)) & 15u), step, lo);
    char* dst = a.rows_out[u.kv] + (long long)u.t * a.row_stride_b[u.kv] + (long long)(u.g * 8 + sub) * (F32 ? 32 : 16);
    if (F32) {
      ((f32x4*)dst)[0] = f32x4{x[0], x[1], x[2], x[3]};
      ((f32x4*)dst)[1] = f32x4{x[4], x[5], x[6], x[7]};
    } else {
      *(u32x4*)dst = u32x4{pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7])};
    }
  }
}

// ---------------------------------------------------------------------------------------------------- decode
// A wave takes one kv head and 64 keys at a time, all by itself (no barriers):
//   S^T = C_k Q^T  in v_mfma_f32_16x16x32_bf16 tiles of 16 keys x 16 query heads, one accumulator per
//         group of 64 elements; lane = one query head and keys 16t + 4*quarter + j;
//   O^T = C_v^T P'^T with P' = weight * step, again one operand per group.
// Codes of eight keys sit in one word; (w >> 4i & 0x000F000F) << 3 | 0x41804180 is two bf16 numbers 16 + code
// (0x4180 = 16.0, whose mantissa has the code's place at bits 3..6), so a pair costs two instructions and
// the 16 goes into the lowest value: lo - 16 step.  The word order that leaves -- elements 0,4,1,5,2,6,3,7 -- is given to
// the other operand as well.  V's codes are transposed by the 4-bit transposing read: 16 lanes point at the rows of
// 16 keys, eight bytes each, and lane i receives column i.
constexpr int kQ4Wave = 64;       // keys per wave and step

// two 16 + code numbers for elements e and e + 4 of a word, e = 0..3
__device__ __forceinline__ unsigned codes_of(unsigned w, int e) {
  const unsigned s = e == 0 ? w << 3 : (w >> (4 * e - 3));
  return (s & 0x00780078u) | 0x41804180u;
}
__device__ __forceinline__ bf16x8 codes8(unsigned w) {
  return __builtin_bit_cast(bf16x8, u32x4{codes_of(w, 0), codes_of(w, 1), codes_of(w, 2), codes_of(w, 3)});
}

template <int D, bool MASS>
__global__ __launch_bounds__(64 * q4_waves(D)) void k_q4_attn(Q4AttnArgs a) {
  constexpr int W = q4_waves(D);
  constexpr int NG = D / kQ4Group;          // groups per head row
  constexpr int HB = D / 2;                 // code bytes of a head row
  constexpr int VROW = HB + 8;              // ... and in LDS: the eight-byte columns of 64 rows spread over the banks
  constexpr int VPIECES = HB / 16;          // 16-byte pieces of a V row
  constexpr int DT = D / 16;
  __shared__ __align__(16) unsigned char sv[W][kQ4Wave * VROW];
  __shared__ __align__(16) f32x2 spair[W][2][NG][kQ4Wave];      // (step, offset) of every key: K's times c, V's
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, quarter = lane >> 4;
  const int r = blockIdx.y;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  const bool one = a.parts * a.wave_parts == 1;      // a single piece: the output is final
  const int qtiles = (a.Gq + 15) / 16;
  const int q16 = (int)(blockIdx.z % qtiles) * 16;   // first query head of the group that this work-group takes
  const int head = a.wave_parts > 1 ? wave / a.wave_parts : (int)(blockIdx.z / qtiles) * W + wave;
  const int wp = wave % a.wave_parts;
  if (head >= a.Hkv) return;
  const int wkeys = a.part_keys / a.wave_parts;
  const long long begin = (long long)blockIdx.x * a.part_keys + (long long)wp * wkeys;
  if (begin >= len && !(one && len == 0)) return;
  const int k_begin = (int)begin, k_end = len - k_begin < wkeys ? len : k_begin + wkeys;

  // ---- queries: lane = query head q16 + l16, element order of the codes
  u32x4 qf[NG][2];
  float qsum[NG];
  const bool live = q16 + l16 < a.Gq;
  {
    const char* src = a.q + (long long)r * a.q_stride_b + (long long)(head * a.Gq + imin(q16 + l16, a.Gq - 1)) * (D * 2);
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
  }

  f32x4 o[DT];
  float m = -INFINITY, l = 0.0f, ol[NG];      // reference, sum of weights, what the groups' offsets add up to
#pragma unroll
  for (int g = 0; g < NG; ++g) ol[g] = 0.0f;
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) o[dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  const long long head_codes = (long long)head * HB, head_pairs = q4_code_bytes(a.Hkv, D) + (long long)head * NG * 4;
  // slot of this lane's key of the step at k0 (keys past the end repeat the last one)
  auto slot_of = [&](int k0) -> int64_t {
    unsigned blk, at;
    divmod_by((unsigned)imin(k0 + lane, len - 1), (unsigned)a.kv_block, a.kv_magic, blk, at);
    return (int64_t)a.block_table[(long long)r * a.table_stride + blk] * a.kv_block + at;
  };
  u32x2 kc[4][NG];                     // K codes: key 16t + l16, elements 64g + 16*quarter ..
  u32x4 vc[VPIECES];                   // V codes: 16-byte pieces of keys in row order
  unsigned kp[NG], vp[NG];             // this lane's key's pairs
  auto fetch = [&](int64_t slot) {
    const int lo = (int)slot, hi = (int)(slot >> 32);
    auto of = [&](int key) { return ((int64_t)__shfl(hi, key) << 32) | (unsigned)__shfl(lo, key); };
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const char* row = a.k + of(16 * t + l16) * a.cache_stride + head_codes + quarter * 8;
#pragma unroll
      for (int g = 0; g < NG; ++g) kc[t][g] = *(const u32x2*)(row + g * 32);
    }
#pragma unroll
    for (int i = 0; i < VPIECES; ++i) {
      const int piece = i * 64 + lane;
      vc[i] = *(const u32x4*)(a.v + of(piece / VPIECES) * a.cache_stride + head_codes + (piece % VPIECES) * 16);
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      kp[g] = *(const unsigned*)(a.k + slot * a.cache_stride + head_pairs + g * 4);
      vp[g] = *(const unsigned*)(a.v + slot * a.cache_stride + head_pairs + g * 4);
    }
  };

  if (k_begin < k_end) fetch(slot_of(k_begin));
  for (int k0 = k_begin; k0 < k_end; k0 += kQ4Wave) {
    // ---- V codes and the pairs into the wave's own LDS
#pragma unroll
    for (int i = 0; i < VPIECES; ++i) {
      const int piece = i * 64 + lane;
      u32x2* dst = (u32x2*)&sv[wave][(piece / VPIECES) * VROW + (piece % VPIECES) * 16];
      dst[0] = u32x2{vc[i].x, vc[i].y};
      dst[1] = u32x2{vc[i].z, vc[i].w};
    }
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const float step = bf16_hi(kp[g]) * a.c;
      spair[wave][0][g][lane] = f32x2{step, fmaf(-16.0f, step, bf16_lo(kp[g]) * a.c)};
      spair[wave][1][g][lane] = f32x2{bf16_hi(vp[g]), fmaf(8.0f, bf16_hi(vp[g]), bf16_lo(vp[g]))};
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // ---- logits in log2 units: x[t][j] of key k0 + 16t + 4*quarter + j
    float x[4][4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8(kc[t][g].x), __builtin_bit_cast(bf16x8, qf[g][0]), acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8(kc[t][g].y), __builtin_bit_cast(bf16x8, qf[g][1]), acc, 0, 0, 0);
        const f32x4* pr = (const f32x4*)&spair[wave][0][g][16 * t + 4 * quarter];
        const f32x4 p01 = pr[0], p23 = pr[1];
        const float add = qsum[g];
        x[t][0] = fmaf(p01.x, acc[0], g == 0 ? p01.y * add : fmaf(p01.y, add, x[t][0]));
        x[t][1] = fmaf(p01.z, acc[1], g == 0 ? p01.w * add : fmaf(p01.w, add, x[t][1]));
        x[t][2] = fmaf(p23.x, acc[2], g == 0 ? p23.y * add : fmaf(p23.y, add, x[t][2]));
        x[t][3] = fmaf(p23.z, acc[3], g == 0 ? p23.w * add : fmaf(p23.w, add, x[t][3]));
      }
      __builtin_amdgcn_sched_barrier(0);      // (keeps the registers of one tile's codes from living beside the next's)
    }
    if (k0 + kQ4Wave < k_end) fetch(slot_of(k0 + kQ4Wave));
    if (MASS && live) {
      float* dst = a.logits + ((long long)r * a.Hq + head * a.Gq + q16 + l16) * a.logit_stride + k0 + 4 * quarter;
#pragma unroll
      for (int t = 0; t < 4; ++t) *(f32x4*)(dst + 16 * t) = f32x4{x[t][0], x[t][1], x[t][2], x[t][3]};
    }
    if (k0 + kQ4Wave > k_end) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (k0 + 16 * t + 4 * quarter + j >= len) x[t][j] = -INFINITY;
    }
    // ---- running softmax (the first key of a step is always there: no row without a maximum)
    float mx = x[0][0];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) mx = fmaxf(mx, x[t][j]);
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    if (__any(mx > m)) {
      const float up = fmaxf(m, mx), f = exp2_of(m - up);
      m = up;
      l *= f;
#pragma unroll
      for (int g = 0; g < NG; ++g) ol[g] *= f;
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
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      bf16x8 pw[2];
#pragma unroll
      for (int mm = 0; mm < 2; ++mm) {
        const f32x4* pa = (const f32x4*)&spair[wave][1][g][32 * mm + 4 * quarter];
        const f32x4* pb = (const f32x4*)&spair[wave][1][g][32 * mm + 16 + 4 * quarter];
        const f32x4 a01 = pa[0], a23 = pa[1], b01 = pb[0], b23 = pb[1];
        const float sa[4] = {a01.x, a01.z, a23.x, a23.z}, la[4] = {a01.y, a01.w, a23.y, a23.w};
        const float sb[4] = {b01.x, b01.z, b23.x, b23.z}, lb[4] = {b01.y, b01.w, b23.y, b23.w};
        unsigned w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float wa = x[2 * mm][j], wb = x[2 * mm + 1][j];
          w[j] = pack2(wa * sa[j], wb * sb[j]);
          // 24 = the 16 of every code and its middle 8 are taken back with the rounded weights that multiplied them, the
          // middle is added with the exact ones: what a weight's rounding multiplies is code - 8, not code + 16
          ol[g] = fmaf(wa, la[j], fmaf(wb, lb[j], ol[g]));
          ol[g] = fmaf(-24.0f, bf16_lo(w[j]) + bf16_hi(w[j]), ol[g]);
        }
        pw[mm] = __builtin_bit_cast(bf16x8, u32x4{w[0], w[1], w[2], w[3]});
      }
#pragma unroll
      for (int dd = 0; dd < 4; ++dd) {
        const int dt = g * 4 + dd;
        typedef int i32x2 __attribute__((ext_vector_type(2)));
        typedef __attribute__((address_space(3))) i32x2* lds2;
        const int row = 16 * (l16 >> 2) + 4 * quarter + (l16 & 3);
        const i32x2 vt = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds2)&sv[wave][row * VROW + dt * 8]);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8((unsigned)vt.x), pw[0], o[dt], 0, 0, 0);
        o[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes8((unsigned)vt.y), pw[1], o[dt], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }

  // ---- o[dt][j]: element 16*dt + 4*quarter + j of query head q16 + l16
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int g = 0; g < NG; ++g) {
    ol[g] += __shfl_xor(ol[g], 16);
    ol[g] += __shfl_xor(ol[g], 32);
  }
  if (!live) return;
  const long long hq = head * a.Gq + q16 + l16;
  if (!one) {
    const long long at = ((long long)r * a.Hq + hq) * (a.parts * a.wave_parts) + blockIdx.x * a.wave_parts + wp;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt) {
      const float b = ol[dt / 4];
      *(f32x4*)(a.o_part + at * D + dt * 16 + quarter * 4) = f32x4{o[dt][0] + b, o[dt][1] + b, o[dt][2] + b, o[dt][3] + b};
    }
    if (quarter == 0) {
      a.ml_part[2 * at] = m;
      a.ml_part[2 * at + 1] = l;
    }
    return;
  }
  const float inv = len > 0 ? 1.0f / l : 0.0f;
  char* dst = a.out + (long long)r * a.out_stride_b + hq * (D * 2);
#pragma unroll
  for (int dt = 0; dt < DT; ++dt) {
    const float b = ol[dt / 4];
    *(u32x2*)(dst + (dt * 16 + quarter * 4) * 2) =
        u32x2{pack2((o[dt][0] + b) * inv, (o[dt][1] + b) * inv), pack2((o[dt][2] + b) * inv, (o[dt][3] + b) * inv)};
  }
  const float lse2 = len > 0 ? m + __log2f(l) : -INFINITY;
  if (quarter == 0 && a.lse != nullptr) a.lse[hq * a.lse_stride + r] = lse2 * 0.69314718055994530942f;
  if (quarter == 0 && MASS) a.lse2[(long long)r * a.Hq + hq] = lse2;
}

// Joins a query head's pieces in order: a wave per (sequence, query head).
template <int D>
__global__ __launch_bounds__(256) void k_q4_join(Q4AttnArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int r = blockIdx.y, hq = blockIdx.x * 4 + wave;
  if (hq >= a.Hq) return;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  const int pieces = a.parts * a.wave_parts, wkeys = a.part_keys / a.wave_parts;
  const int live = (len + wkeys - 1) / wkeys;      // pieces hold consecutive runs of keys
  constexpr int PER = D / 64;
  const long long at0 = ((long long)r * a.Hq + hq) * pieces;
  float m = -INFINITY;
  for (int p = lane; p < live; p += 64) m = fmaxf(m, a.ml_part[2 * (at0 + p)]);
  for (int d = 1; d < 64; d <<= 1) m = fmaxf(m, __shfl_xor(m, d));
  float l = 0.0f, acc[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) acc[i] = 0.0f;
  for (int p = 0; p < live; ++p) {
    const long long at = at0 + p;
    const float f = exp2_of(a.ml_part[2 * at] - m);
    l = fmaf(a.ml_part[2 * at + 1], f, l);
#pragma unroll
    for (int i = 0; i < PER; ++i) acc[i] = fmaf(a.o_part[at * D + lane * PER + i], f, acc[i]);
  }
  const float inv = len > 0 ? 1.0f / l : 0.0f;
  __bf16* dst = (__bf16*)(a.out + (long long)r * a.out_stride_b + (long long)hq * (D * 2));
#pragma unroll
  for (int i = 0; i < PER; ++i) dst[lane * PER + i] = (__bf16)(acc[i] * inv);
  const float lse2 = len > 0 ? m + __log2f(l) : -INFINITY;
  if (lane == 0 && a.lse != nullptr) a.lse[(long long)hq * a.lse_stride + r] = lse2 * 0.69314718055994530942f;
  if (lane == 0 && a.lse2 != nullptr) a.lse2[(long long)r * a.Hq + hq] = lse2;
}

// Accumulated weight: the query heads' weights of a token added in order, their mean onto what it had.
__global__ __launch_bounds__(256) void k_q4_mass(Q4AttnArgs a) {
  const int r = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  const int len = imin(imax(a.kv_len[r], 0), a.max_len);
  if (i >= len) return;
  const float* x = a.logits + (long long)r * a.Hq * a.logit_stride + i;
  float sum = 0.0f;
  for (int h = 0; h < a.Hq; ++h) sum += exp2_of(x[h * a.logit_stride] - a.lse2[(long long)r * a.Hq + h]);
  const long long at = (long long)r * a.mass_stride + i;
  a.mass_out[at] = (a.mass_in != nullptr ? a.mass_in[at] : 0.0f) + sum / (float)a.Hq;
}

template <int D>
hipError_t launch_q4_attn(const Q4AttnArgs& a, hipStream_t s) {
  const dim3 grid(a.parts, a.R, a.head_groups * ((a.Gq + 15) / 16)), block(64 * q4_waves(D));
  if (a.mass_out != nullptr) hipLaunchKernelGGL((k_q4_attn<D, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_q4_attn<D, false>), grid, block, 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.parts * a.wave_parts > 1) {
    hipLaunchKernelGGL((k_q4_join<D>), dim3((a.Hq + 3) / 4, a.R), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.mass_out != nullptr && a.max_len > 0) {
    hipLaunchKernelGGL(k_q4_mass, dim3((a.max_len + 255) / 256, a.R), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_q4_store(const Q4CopyArgs& a, bool f32, hipStream_t s) {
  const dim3 grid((unsigned)((a.n + kQ4Rows - 1) / kQ4Rows));
  if (f32) hipLaunchKernelGGL((k_q4_store<true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_q4_store<false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_q4_load(const Q4CopyArgs& a, bool f32, hipStream_t s) {
  const dim3 grid((unsigned)((a.n + kQ4Rows - 1) / kQ4Rows));
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
