// Launchers of the attention layer's kernels: causal attention of a packed batch, the 4-bit KV
// cache with its decode attention, and eviction from a paged cache (internal header).
#pragma once

#include "up_common.h"
#include "up_kernels.h"

namespace up {

// --- causal attention of a packed batch
// pieces of part_keys keys that `keys` keys are cut into (both below 2^31: their sum leaves an int, not 32 bits)
UP_HD int attn_pieces(int keys, int part_keys) { return (int)(((unsigned)keys + (unsigned)part_keys - 1u) / (unsigned)part_keys); }

struct AttnArgs {
  const char* q;
  const char* k;
  const char* v;
  char* out;
  float* lse;                      // [Hq][lse_stride] natural log, or nullptr
  const int32_t* cu;
  const int32_t* cu_k;             // == cu when no sequence has earlier context
  const int32_t* block_table;      // paged keys and values, or nullptr
  long long table_stride;
  int kv_block;
  unsigned kv_magic;               // 0xFFFFFFFF / kv_block
  long long q_stride_b, k_stride_b, v_stride_b, out_stride_b;
  long long lse_stride;
  float c;                         // scale * log2(e)
  int R, Hq, Hkv, Gq;
  int rows;                        // query rows (token x query head of one kv head) per work-group: 256 or 128
  int slots;                       // row tiles of all sequences (an upper bound)
  int items;                       // work-groups per kv head: row tiles, or their pieces along the keys
  int part_keys;                   // keys per work-group when the key axis is split, else 0
  int parts;                       // pieces of the longest sequence
  int32_t* base;                   // [slots] first piece of a row tile that is cut, -1 for one that is not
  float* o_part;                   // [pieces][Hkv][rows][D] sums of weighted values
  float* ml_part;                  // [pieces][Hkv][rows] pairs (reference in log2 units, sum of weights)
};

// --- the 4-bit KV cache
// waves of a decode work-group, each on a kv head (D = 256: four, with twice the registers)
constexpr UP_HD int q4_waves(int D) { return D == 256 ? 4 : 8; }
constexpr int kQ4MaxWaveParts = 4;       // waves of a work-group that may share a kv head's keys
constexpr int kQ4JoinWaves = 16;         // waves that join the pieces of a query head, at most
// ... and waves per SIMD that its registers are held to
constexpr UP_HD int q4_dense(int D) { return D == 64 ? 4 : D == 128 ? 2 : 1; }
constexpr int kQ4Group = 64;        // elements that share one (lowest value, step) pair
UP_HD long long q4_code_bytes(int heads, int D) { return (long long)heads * D / 2; }
UP_HD long long q4_row_bytes(int heads, int D) { return q4_code_bytes(heads, D) + (long long)heads * (D / kQ4Group) * 4; }

struct Q4CopyArgs {                 // rows <-> slots of the cache, for keys and values
  const char* rows_in[2];           // store: rows to quantise (nullptr: none)
  char* rows_out[2];                // load: rows to write
  char* cache[2];
  long long row_stride_b[2];        // bytes between rows
  long long cache_stride;           // bytes between slots
  const int64_t* slots;
  const int32_t* count_dev;         // rows t < count_dev[0] when given
  long long n, num_slots;
  int heads, D;
};

struct Q4AttnArgs {
  const char* q;
  const char* k;
  const char* v;
  char* out;
  float* lse;
  const int32_t* kv_len;
  const int32_t* block_table;
  long long table_stride, cache_stride, q_stride_b, out_stride_b, lse_stride;
  const float* mass_in;
  float* mass_out;
  long long mass_stride;
  int kv_block;
  unsigned kv_magic;
  float c;
  int R, Hq, Hkv, Gq, D, max_len;
  int groups;                       // work-groups along the keys of all sequences
  int head_groups;                  // ... times these: q4_waves kv heads each
  int wave_parts;                   // waves of a work-group that share a kv head, each with 64 keys of a step
  unsigned* seq_step;               // [R + 1] first step of every sequence in the row of all steps
  float* o_part;                    // [groups + R][wave_parts][Hq][D]
  float* ml_part;                   // [groups + R][wave_parts][Hq] pairs
  float* lse2;                      // [R][Hq] normaliser in log2 units, for the accumulated weights
  float* logits;                    // [R][Hq][logit_stride] in log2 units
  long long logit_stride;
};

// --- eviction from a paged cache
struct EvictArgs {
  char* k;
  char* v;
  long long row_bytes, cache_stride;
  const float* mass;
  float* mass_out;
  long long mass_stride, mass_out_stride;
  const int32_t* kv_len;
  const int32_t* block_table;
  const int32_t* new_table;
  long long table_stride, new_table_stride;
  int32_t* kept_idx;                // [R][mass_out_stride]
  int32_t* new_len;
  int R, max_len, budget, n_sink, n_recent, kv_block;
  unsigned kv_magic, piece_magic;   // 0xFFFFFFFF / kv_block, 0xFFFFFFFF / (row_bytes / 16)
};

#if defined(__HIPCC__)
hipError_t launch_attention(const AttnArgs& a, bool f32, int D, hipStream_t s);
hipError_t launch_q4_store(const Q4CopyArgs& a, bool f32, hipStream_t s);
hipError_t launch_q4_load(const Q4CopyArgs& a, bool f32, hipStream_t s);
hipError_t launch_q4_attention(const Q4AttnArgs& a, hipStream_t s);
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);

// An entry of a block table at an index that is the same for the whole wave.  No kernel writes a table, so it may come through the
// scalar cache: its wait is then not one for the vector loads in flight.
__device__ __forceinline__ int table_entry(const int32_t* table, unsigned i) {
  return ((const __attribute__((address_space(4))) int32_t*)table)[i];
}

// x -> (x / d, x % d) with a precomputed magic = 0xFFFFFFFF / d  (x < 2^31)
__device__ __forceinline__ void divmod_by(unsigned x, unsigned d, unsigned magic, unsigned& qo, unsigned& ro) {
  unsigned qq = __umulhi(x, magic);
  unsigned rr = x - qq * d;
  if (rr >= d) { ++qq; rr -= d; }
  qo = qq;
  ro = rr;
}
#else
// the host-only build of the argument checks has no kernels to launch
inline hipError_t launch_attention(const AttnArgs&, bool, int, hipStream_t) { return hipSuccess; }
inline hipError_t launch_q4_store(const Q4CopyArgs&, bool, hipStream_t) { return hipSuccess; }
inline hipError_t launch_q4_load(const Q4CopyArgs&, bool, hipStream_t) { return hipSuccess; }
inline hipError_t launch_q4_attention(const Q4AttnArgs&, hipStream_t) { return hipSuccess; }
inline hipError_t launch_evict(const EvictArgs&, hipStream_t) { return hipSuccess; }
#endif

}  // namespace up
