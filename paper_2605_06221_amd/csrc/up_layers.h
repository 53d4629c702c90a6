// Launchers of the operators that the layers between two drops are made of: linear attention with a decay, norm and
// rotation of query and key heads, pages for new tokens (internal header).
#pragma once

#include "up_common.h"

namespace up {

// --- linear attention
struct LinearArgs {
  const char* q;
  const char* k;
  const char* v;
  char* out;
  const float* log_decay;          // [Hkv]
  const int32_t* cu;
  float* states;                   // slots of [Hkv][D][D], or nullptr
  long long state_stride;          // elements between slots
  const int32_t* state_in;         // [R] slot that a sequence starts from (nullptr, or outside the pool: from zero)
  const int32_t* state_out;        // [R] slot that its state is stored to (nullptr, or outside the pool: not stored)
  long long num_states;
  long long q_stride_b, k_stride_b, v_stride_b, out_stride_b;
  float scale;
  int R, Hq, Hkv, Gq;
  int piece;                       // tokens of a piece (a multiple of 32); longer sequences are cut
  int slots;                       // pieces of all sequences (an upper bound)
  float* adds;                     // [2 T / piece + 1][Hkv][D][D] what the pieces of cut sequences add to the state; nullptr: none is cut
};

// --- norm and rotation
struct RotateArgs {
  const char* in[3];               // queries, keys, values; nullptr: not there
  char* out[3];
  long long in_stride_b[3], out_stride_b[3];
  const char* weight[2];           // of queries, keys; nullptr: 1
  const int32_t* pos;
  const float* inv_freq;
  const int64_t* slots;            // rows of keys and values in their outputs; nullptr: the tokens' own
  const int32_t* count_dev;
  long long n, num_slots;
  float eps;                       // 0: rows are not normalised
  int heads[3];                    // 0 where a tensor is not there
  int D, rot;
  int pairs;
  int waves;                       // waves that share a token
  int stream;                      // more bytes than the last-level cache holds
};

// --- pages for new tokens
struct PagesArgs {
  const int32_t* kv_len;
  const int32_t* num_new;
  const int32_t* dropped;          // [R] tokens of a sequence that the cache does not hold; nullptr: none
  const int32_t* free_pages;
  const int32_t* num_free;
  int32_t* block_table;
  long long table_stride;
  int32_t* free_left;
  int32_t* new_len;
  int32_t* cu;
  int32_t* cu_k;
  int32_t* pos;
  int64_t* slots;
  int32_t* served;
  long long capacity;
  int R, kv_block;
  unsigned kv_magic;               // 0xFFFFFFFF / kv_block
  int one_launch;
};

#if defined(__HIPCC__)
hipError_t launch_linear(const LinearArgs& a, bool f32, int D, hipStream_t s);
hipError_t launch_linear_step(const LinearArgs& a, bool f32, int D, hipStream_t s);
hipError_t launch_rotate(const RotateArgs& a, bool f32, hipStream_t s);
hipError_t launch_pages(const PagesArgs& a, hipStream_t s);
#else
// the host-only build of the argument checks has no kernels to launch
inline hipError_t launch_linear(const LinearArgs&, bool, int, hipStream_t) { return hipSuccess; }
inline hipError_t launch_linear_step(const LinearArgs&, bool, int, hipStream_t) { return hipSuccess; }
inline hipError_t launch_rotate(const RotateArgs&, bool, hipStream_t) { return hipSuccess; }
inline hipError_t launch_pages(const PagesArgs&, hipStream_t) { return hipSuccess; }
#endif

}  // namespace up
