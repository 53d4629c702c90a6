// Linear attention with a decay for each kv head (lam = exp(log_decay), at most 1):
//     S_t = lam S_{t-1} + k_t^T v_t,        out_t = scale q_t S_t      (S: D x D, float, carried by the sequence)
//
// k_linear_tokens, token after token: a work-group holds 32 columns of a head's state in registers, eight lanes by 32 groups of rows.
#include "up_layers.h"

namespace up {

__device__ __forceinline__ float linear_load(const char* p, int i, bool f32) {
  return f32 ? ((const float*)p)[i] : __builtin_bit_cast(float, (unsigned)((const unsigned short*)p)[i] << 16);
}

// exp(log_decay * n) as the sum of two floats: a state is scaled once per step, and the error of one float would add up over the steps
__device__ __forceinline__ void linear_decay(float log_decay, int n, float& hi, float& lo) {
  const double x = exp((double)fminf(fmaxf(log_decay, -1e4f), 0.0f) * (double)n);
  hi = (float)x;
  lo = (float)(x - (double)hi);
}

__device__ __forceinline__ long long linear_slot(const int32_t* of, int r, long long num) {
  if (of == nullptr) return -1;
  const long long s = of[r];
  return s >= 0 && s < num ? s : -1;
}

template <bool F32, int D>
__global__ __launch_bounds__(256) void k_linear_tokens(LinearArgs a) {
  constexpr int SLICES = D / 32, PER = D / 32, E = F32 ? 4 : 2;      // rows of the state per lane
  const int slice = blockIdx.x % SLICES, kvh = (blockIdx.x / SLICES) % a.Hkv, r = blockIdx.x / (SLICES * a.Hkv);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int col = slice * 32 + (lane & 7) * 4, row0 = (wave * 8 + (lane >> 3)) * PER;
  __shared__ f32x4 part[2][4][8];
  const int c0 = a.cu != nullptr ? a.cu[r] : r, N = a.cu != nullptr ? a.cu[r + 1] - c0 : 1;
  const long long from = linear_slot(a.state_in, r, a.num_states), to = linear_slot(a.state_out, r, a.num_states);
  f32x4 S[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    S[i] = f32x4{0, 0, 0, 0};
    if (from >= 0) S[i] = *(const f32x4*)(a.states + from * a.state_stride + ((long long)kvh * D + row0 + i) * D + col);
  }
  float hi, lo;
  linear_decay(a.log_decay[kvh], 1, hi, lo);
  int turn = 0;
  for (int t = c0; t < c0 + N; ++t) {
    const char* k = a.k + (long long)t * a.k_stride_b + (long long)kvh * D * E;
    const char* v = a.v + (long long)t * a.v_stride_b + (long long)kvh * D * E;
    f32x4 v4;
#pragma unroll
    for (int i = 0; i < 4; ++i) v4[i] = linear_load(v, col + i, F32);
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const float ki = linear_load(k, row0 + i, F32);
#pragma unroll
      for (int e = 0; e < 4; ++e) S[i][e] = fmaf(ki, v4[e], fmaf(S[i][e], hi, S[i][e] * lo));
    }
    for (int g = 0; g < a.Gq; ++g, turn ^= 1) {
      const int h = kvh * a.Gq + g;
      const char* q = a.q + (long long)t * a.q_stride_b + (long long)h * D * E;
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
      if (lane < 8) part[turn][wave][lane] = o;
      __syncthreads();      // (two buffers: the readers of this one are through before it is written again)
      if (tid < 8) {
        const f32x4 p0 = part[turn][0][tid], p1 = part[turn][1][tid], p2 = part[turn][2][tid], p3 = part[turn][3][tid];
        char* dst = a.out + (long long)t * a.out_stride_b + (long long)h * D * E;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float y = ((p0[e] + p1[e]) + (p2[e] + p3[e])) * a.scale;
          if (F32) ((float*)dst)[col + e] = y;
          else ((__bf16*)dst)[col + e] = (__bf16)y;
        }
      }
    }
  }
  if (to >= 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) *(f32x4*)(a.states + to * a.state_stride + ((long long)kvh * D + row0 + i) * D + col) = S[i];
  }
}

template <bool F32, int D>
static hipError_t launch_linear_tokens_form(const LinearArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((k_linear_tokens<F32, D>), dim3((unsigned)a.R * a.Hkv * (D / 32)), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_linear_tokens(const LinearArgs& a, bool f32, int D, hipStream_t s) {
  if (f32) return D == 64 ? launch_linear_tokens_form<true, 64>(a, s) : launch_linear_tokens_form<true, 128>(a, s);
  return D == 64 ? launch_linear_tokens_form<false, 64>(a, s) : D == 128 ? launch_linear_tokens_form<false, 128>(a, s)
                                                                         : launch_linear_tokens_form<false, 256>(a, s);
}

}  // namespace up
