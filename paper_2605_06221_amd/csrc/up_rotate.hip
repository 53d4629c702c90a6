// Norm of query and key heads and rotation by the token's position, in one pass, keys and values straight into the slots of a
// paged cache.
//
// A head row x of D elements becomes  y = x / sqrt(mean x^2 + eps) * weight  and of y each pair (a, b) of the first rot
// elements  (a cos - b sin, b cos + a sin)  by the angle position * inv_freq[pair].
//
// Bound by memory: every row is read and written once (32768 tokens, 40/8 heads of 128, values copied along: 197 us, 4.8 TB/s, 95 % of a
// copy's rate).  A lane holds 32 bytes of a row, the 16 of the pairs' first halves and the 16 of
// their partners (the pairs are then a lane's own business), and the lanes of a head add up its squares.  A token's heads share its
// angles: lane f of a wave takes pair f's turn in double (a position of 10^5 times 1 rad leaves nothing of a float's angle) and the others fetch
// its sine and cosine.
#include "up_layers.h"

namespace up {

template <bool F32>
struct RotateLane {
  static constexpr int VE = F32 ? 4 : 8;      // elements of 16 bytes
};

template <bool F32>
__device__ __forceinline__ void rotate_unpack(const u32x4& w, float* x) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const unsigned u = w[i];
    if (F32) {
      x[i] = __builtin_bit_cast(float, u);
    } else {
      x[2 * i] = __builtin_bit_cast(float, u << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, u & 0xFFFF0000u);
    }
  }
}
template <bool F32>
__device__ __forceinline__ u32x4 rotate_pack(const float* x) {
  u32x4 w;
  if (F32) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(unsigned, x[i]);
  } else {
    typedef float f32x8 __attribute__((ext_vector_type(8)));
    f32x8 v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = x[i];
    w = __builtin_bit_cast(u32x4, __builtin_convertvector(v, bf16x8));
  }
  return w;
}

// STREAM: more than the last-level cache holds, so that rows are read and written past it
template <bool STREAM>
__device__ __forceinline__ u32x4 rotate_load(const char* p) { return STREAM ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p; }
template <bool STREAM>
__device__ __forceinline__ void rotate_store(u32x4 x, char* p) {
  if (STREAM) __builtin_nontemporal_store(x, (u32x4*)p);
  else *(u32x4*)p = x;
}

template <bool F32, int D, bool STREAM>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a) {
  constexpr int VE = RotateLane<F32>::VE, LPH = D / (2 * VE), HPW = 64 / LPH, E = F32 ? 4 : 2;
  const int lane = threadIdx.x & 63;
  const long long wave = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const long long t = wave / a.waves;
  const int part = (int)(wave % a.waves);
  if (t >= a.n || (a.count_dev != nullptr && t >= (long long)a.count_dev[0])) return;
  // ---- where a lane's elements lie, and which pairs' angles they need
  const int j = lane % LPH, half = a.rot / 2;
  int ea, eb;
  bool turns;
  if (a.pairs) {
    ea = 2 * VE * j;
    eb = ea + VE;
    turns = ea < a.rot;
  } else {
    turns = VE * j < half;
    ea = turns ? VE * j : 2 * VE * j;
    eb = turns ? half + VE * j : ea + VE;
  }
  float c[VE], s[VE];
  if (a.rot > 0) {
    const double p = (double)a.pos[t];
    float cl[D / 128 + 1], sl[D / 128 + 1];
#pragma unroll
    for (int i = 0; i < (D == 256 ? 2 : 1); ++i) {
      const int f = lane + 64 * i;
      const double turn = f < half ? p * (double)a.inv_freq[f] * 0.15915494309189533577 : 0.0;      // 1 / 2 pi
      sincospif(2.0f * (float)(turn - rint(turn)), &sl[i], &cl[i]);
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      const int f = VE * j + e;
      c[e] = __shfl(cl[0], f & 63);
      s[e] = __shfl(sl[0], f & 63);
      if (D == 256) {
        const float c1 = __shfl(cl[1], f & 63), s1 = __shfl(sl[1], f & 63);
        if (f >= 64) { c[e] = c1; s[e] = s1; }
      }
    }
  }
  if (a.rot == 0 || !turns) {
#pragma unroll
    for (int e = 0; e < VE; ++e) { c[e] = 1.0f; s[e] = 0.0f; }
  }
  const long long slot = a.slots != nullptr ? a.slots[t] : t;
  const bool kept = a.slots == nullptr || (slot >= 0 && slot < a.num_slots);
  const int rotated = a.heads[0] + a.heads[1], all = rotated + a.heads[2];
  u32x4 weight[2][2];      // of queries, keys: the lane's elements
  const bool weighted[2] = {a.weight[0] != nullptr, a.weight[1] != nullptr};
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    weight[which][0] = weight[which][1] = u32x4{0, 0, 0, 0};
    if (weighted[which]) {
      weight[which][0] = *(const u32x4*)(a.weight[which] + ea * E);
      weight[which][1] = *(const u32x4*)(a.weight[which] + eb * E);
    }
  }
  // two rounds' rows are under way together
  for (int h0 = part * HPW; h0 < all; h0 += 2 * a.waves * HPW) {
    u32x4 wa[2], wb[2];
    int type[2];
    long long offset[2];
    bool live[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int hh = h0 + i * a.waves * HPW + lane / LPH;
      live[i] = hh < all;
      type[i] = hh < a.heads[0] ? 0 : hh < rotated ? 1 : 2;
      offset[i] = (long long)(type[i] == 0 ? hh : type[i] == 1 ? hh - a.heads[0] : hh - rotated) * (D * E);
      wa[i] = wb[i] = u32x4{0, 0, 0, 0};
      if (live[i]) {
        const char* src = a.in[type[i]] + t * a.in_stride_b[type[i]] + offset[i];
        wa[i] = rotate_load<STREAM>(src + ea * E);
        wb[i] = rotate_load<STREAM>(src + eb * E);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      // (elements that are neither normalised nor turned stay as they are: a turn by nothing would lose the sign of a zero)
      if (type[i] < 2 && (turns || a.eps > 0.0f)) {
        float x[VE], y[VE];
        rotate_unpack<F32>(wa[i], x);
        rotate_unpack<F32>(wb[i], y);
        if (a.eps > 0.0f) {
          float sum = 0.0f;
#pragma unroll
          for (int e = 0; e < VE; ++e) sum = fmaf(x[e], x[e], fmaf(y[e], y[e], sum));
#pragma unroll
          for (int d = 1; d < LPH; d <<= 1) sum += __shfl_xor(sum, d);
          const float inv = 1.0f / sqrtf(sum * (1.0f / D) + a.eps);
          float wx[VE], wy[VE];
          rotate_unpack<F32>(type[i] == 0 ? weight[0][0] : weight[1][0], wx);
          rotate_unpack<F32>(type[i] == 0 ? weight[0][1] : weight[1][1], wy);
          const bool use = type[i] == 0 ? weighted[0] : weighted[1];
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            x[e] *= use ? inv * wx[e] : inv;
            y[e] *= use ? inv * wy[e] : inv;
          }
        }
        float u[VE], w[VE];
        if (a.pairs) {      // the lane's elements in a row: x then y, neighbours are pairs
#pragma unroll
          for (int e = 0; e < VE; e += 2) {
            u[e] = x[e] * c[e / 2] - x[e + 1] * s[e / 2];
            u[e + 1] = x[e + 1] * c[e / 2] + x[e] * s[e / 2];
            w[e] = y[e] * c[VE / 2 + e / 2] - y[e + 1] * s[VE / 2 + e / 2];
            w[e + 1] = y[e + 1] * c[VE / 2 + e / 2] + y[e] * s[VE / 2 + e / 2];
          }
        } else {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            u[e] = x[e] * c[e] - y[e] * s[e];
            w[e] = y[e] * c[e] + x[e] * s[e];
          }
        }
        wa[i] = rotate_pack<F32>(u);
        wb[i] = rotate_pack<F32>(w);
      }
      if (live[i] && (type[i] == 0 || kept)) {
        char* dst = a.out[type[i]] + (type[i] == 0 ? t : slot) * a.out_stride_b[type[i]] + offset[i];
        rotate_store<STREAM>(wa[i], dst + ea * E);
        rotate_store<STREAM>(wb[i], dst + eb * E);
      }
    }
  }
}

template <bool F32, int D>
static hipError_t launch_rotate_form(const RotateArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((a.n * a.waves + 3) / 4));
  if (a.stream) hipLaunchKernelGGL((k_rotate<F32, D, true>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((k_rotate<F32, D, false>), grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_rotate(const RotateArgs& a, bool f32, hipStream_t s) {
  if (f32) return a.D == 64 ? launch_rotate_form<true, 64>(a, s) : launch_rotate_form<true, 128>(a, s);
  return a.D == 64 ? launch_rotate_form<false, 64>(a, s) : a.D == 128 ? launch_rotate_form<false, 128>(a, s) : launch_rotate_form<false, 256>(a, s);
}

}  // namespace up
