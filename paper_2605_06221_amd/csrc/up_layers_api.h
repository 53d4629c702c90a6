// Entry points of the operators that the layers between two drops are made of (windowed attention, linear attention, norm and
// rotation, pages for new tokens): argument checks and launch geometry, host code only.  Part of up_api.hip, behind the
// attention layer's entry points, whose checks it uses.
#pragma once

#include "up_layers.h"

namespace {

int check_window(int32_t window, int32_t n_sink, AttnWindow* w) {
  if (window < 1 || n_sink < 0) return UP_ERR_RANGE;
  *w = AttnWindow{window, n_sink};
  return UP_OK;
}

// ---- linear attention
int linear_args(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride, const float* log_decay,
                float* states, int64_t state_stride, int64_t num_states, const int32_t* state_in, const int32_t* state_out,
                void* out, int64_t out_row_stride, Problem* pb, LinearArgs* a) {
  int st = check_params(p, true, false, pb);
  if (st != UP_OK) return st;
  if (pb->T > 0 && (!q || !k || !v || !out)) return UP_ERR_NULL;
  if (pb->R > 0 && !log_decay) return UP_ERR_NULL;
  const bool any_state = state_in != nullptr || state_out != nullptr;
  if (any_state && pb->R > 0 && num_states > 0 && !states) return UP_ERR_NULL;
  if (num_states < 0) return UP_ERR_SHAPE;
  const int64_t state = (int64_t)pb->Hkv * pb->head_dim * pb->head_dim;
  if (any_state && num_states > 0 && state_stride < state) return UP_ERR_SHAPE;
  const int e = pb->qk_is_f32 ? 4 : 2;
  if ((st = check_row_stride(v_row_stride, pb->Hkv, pb->head_dim, e)) != UP_OK) return st;
  if ((st = check_row_stride(out_row_stride, pb->Hq, pb->head_dim, e)) != UP_OK) return st;
  if (any_state && num_states > 0 && state_stride > kMostStride / num_states) return UP_ERR_UNSUPPORTED;
  // (offsets of a chunk's rows stay within 32 bits)
  if (pb->q_stride * e > kMaxRowStride || pb->k_stride * e > kMaxRowStride || v_row_stride * e > kMaxRowStride ||
      out_row_stride * e > kMaxRowStride)
    return UP_ERR_UNSUPPORTED;
  if (any_state && num_states > 0 && state_stride % 4 != 0) return UP_ERR_ALIGN;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(states)) return UP_ERR_ALIGN;
  if (!aligned_to(log_decay, 4) || !aligned_to(state_in, 4) || !aligned_to(state_out, 4)) return UP_ERR_ALIGN;
  *a = LinearArgs{};
  a->q = (const char*)q; a->k = (const char*)k; a->v = (const char*)v; a->out = (char*)out; a->log_decay = log_decay;
  a->states = states; a->state_stride = state_stride; a->state_in = state_in; a->state_out = state_out; a->num_states = num_states;
  a->q_stride_b = pb->q_stride * e; a->k_stride_b = pb->k_stride * e; a->v_stride_b = v_row_stride * e;
  a->out_stride_b = out_row_stride * e;
  a->scale = pb->scale;
  a->R = pb->R; a->Hq = pb->Hq; a->Hkv = pb->Hkv; a->Gq = pb->Gq;
  // (work-items of a launch are counted in 32 bits)
  if ((int64_t)pb->R * pb->Hkv > (int64_t)(UINT32_MAX / 256) / (pb->head_dim / 32)) return UP_ERR_UNSUPPORTED;
  return UP_OK;
}

// Sequences are cut into pieces of so many tokens that the batch makes a work-group for every place that the CUs have (three a CU; two for 128-wide
// heads that share a state, whose parts fill the registers; one where head rows of 512 bytes fill the LDS), none shorter than two chunks.
// Measured, as pieces of a third, as these, as twice the size: 32768 tokens, 32/8 heads of 128, 309, 250, 270 us (two, three, four places a CU);
// 64 wide, 40/8, ragged 184, 143, 156 (four, three, two); four and six places for all that is 64 wide: ragged 139 -> 153, 153, 32768 tokens of 32/8
// 129 -> 132, 145, 8000 of 8/8 30 -> 37, 36, 16 x 2048 of 40/8 196 -> 184, 173.  Shortest piece of 256 and of 64 tokens: 1000 tokens, 8/8 heads of 128,
// 34 and 23 us, 200 tokens of 32/8 heads of 64 29 and 21.  (Tokens and kv heads are all that the rule looks at.  How many query heads share a state, and
// with it how long a piece takes, is not in it: the last of the 64-wide batches would gain 12 % from six places, where the others lose.)
struct LinearGeometry {
  int piece;
  long long slots;
  size_t total;
};
int linear_geometry(const Problem& pb, const int32_t* cu, LinearGeometry* g) {
  if (pb.T > 1 << 30) return UP_ERR_UNSUPPORTED;      // (a piece past the end of the last sequence is still counted in 31 bits)
  const int places = pb.head_dim * (pb.qk_is_f32 ? 4 : 2) == 512 ? 1 : pb.head_dim == 128 && pb.Gq > 1 ? 2 : 3;
  long long piece = ((long long)pb.T * pb.Hkv / (places * kCUs) + 63) / 64 * 64;
  if (piece < 64) piece = 64;
  g->piece = (int)piece;
  g->slots = pb.T / piece + pb.R;
  g->total = 0;
  for (int r = 0; r < pb.R; ++r)
    if (cu[r + 1] - cu[r] > piece) g->total = (size_t)(2ll * pb.T / piece + 1) * pb.Hkv * pb.head_dim * pb.head_dim * sizeof(float);
  // (work-items of a launch are counted in 32 bits)
  if (piece > INT32_MAX / 2 || g->slots * pb.Hkv > (long long)UINT32_MAX / (2 * pb.head_dim) ||
      (long long)pb.R * pb.Hkv > (long long)(UINT32_MAX / 256) / (pb.head_dim * pb.head_dim / 1024))
    return UP_ERR_UNSUPPORTED;
  return UP_OK;
}

// ---- pages for new tokens
int append_pages_impl(const int32_t* kv_len_dev, const int32_t* num_new_dev, const int32_t* num_dropped_dev, int32_t num_seqs, int32_t kv_block_size,
                      int32_t* block_table, int64_t block_table_stride, const int32_t* free_pages, const int32_t* num_free_dev,
                      int32_t* free_left_dev, int32_t* new_len_dev, int32_t* cu_seqlens_dev, int32_t* cu_seqlens_k_dev, int32_t* pos,
                      int64_t* slots, int64_t capacity, int32_t* num_served_dev, void* stream) {
  if (num_seqs < 0 || capacity < 0) return UP_ERR_SHAPE;
  if (kv_block_size < 1 || block_table_stride < 0) return UP_ERR_RANGE;
  if (!num_free_dev || !free_left_dev || !cu_seqlens_dev || !cu_seqlens_k_dev || !num_served_dev) return UP_ERR_NULL;
  if (num_seqs > 0 && (!kv_len_dev || !num_new_dev || !new_len_dev || !free_pages || (block_table_stride > 0 && !block_table))) return UP_ERR_NULL;
  if (capacity > 0 && (!pos || !slots)) return UP_ERR_NULL;
  if (!aligned_to(kv_len_dev, 4) || !aligned_to(num_new_dev, 4) || !aligned_to(num_dropped_dev, 4) || !aligned_to(block_table, 4) || !aligned_to(free_pages, 4) ||
      !aligned_to(num_free_dev, 4) || !aligned_to(free_left_dev, 4) || !aligned_to(new_len_dev, 4) || !aligned_to(cu_seqlens_dev, 4) ||
      !aligned_to(cu_seqlens_k_dev, 4) || !aligned_to(pos, 4) || !aligned_to(slots, 8) || !aligned_to(num_served_dev, 4))
    return UP_ERR_ALIGN;
  if (capacity > INT32_MAX - 65536 || num_seqs > INT32_MAX - 65536) return UP_ERR_UNSUPPORTED;
  // the lengths may be updated in place, and so may the count of free pages; they overlap in no other way
  const intptr_t apart = (intptr_t)new_len_dev - (intptr_t)kv_len_dev, ends = (intptr_t)num_seqs * (intptr_t)sizeof(int32_t);
  if (apart != 0 && apart > -ends && apart < ends) return UP_ERR_UNSUPPORTED;
  PagesArgs a{};
  a.kv_len = kv_len_dev; a.num_new = num_new_dev; a.dropped = num_dropped_dev; a.free_pages = free_pages; a.num_free = num_free_dev;
  a.block_table = block_table; a.table_stride = block_table_stride; a.free_left = free_left_dev; a.new_len = new_len_dev;
  a.cu = cu_seqlens_dev; a.cu_k = cu_seqlens_k_dev; a.pos = pos; a.slots = slots; a.served = num_served_dev;
  a.capacity = capacity; a.R = num_seqs; a.kv_block = kv_block_size;
  a.kv_magic = 0xFFFFFFFFu / (unsigned)kv_block_size;
  return launch_pages(a, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

}  // namespace

extern "C" {

int uniprefill_attention_window_plan(const up_params* p, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k_host,
                                     int32_t window, int32_t n_sink, size_t* workspace_bytes) {
  AttnWindow w;
  const int st = check_window(window, n_sink, &w);
  return st != UP_OK ? st : attention_plan_impl(p, cu_seqlens_host, cu_seqlens_k_host, &w, workspace_bytes);
}

int uniprefill_attention_window(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride,
                                const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host,
                                const int32_t* cu_seqlens_k_dev, const int32_t* cu_seqlens_k_host,
                                const int32_t* block_table, int64_t block_table_stride, int32_t kv_block_size,
                                int32_t window, int32_t n_sink, void* out, int64_t out_row_stride, float* lse_out,
                                int64_t lse_row_stride, void* workspace, size_t workspace_bytes, void* stream) {
  AttnWindow w;
  const int st = check_window(window, n_sink, &w);
  if (st != UP_OK) return st;
  return attention_impl(p, q, k, v, v_row_stride, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                        PagedKeys{block_table, block_table_stride, kv_block_size}, &w, out, out_row_stride, lse_out, lse_row_stride,
                        workspace, workspace_bytes, stream);
}

int uniprefill_attention_window_step_plan(const up_params* p, int32_t max_kv_len, int32_t window, int32_t n_sink,
                                          size_t* workspace_bytes) {
  Problem pb;
  AttnWindow w;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (workspace_bytes == nullptr) return UP_ERR_NULL;
  if (pb.T != pb.R || max_kv_len < 0) return UP_ERR_SHAPE;
  if ((st = check_window(window, n_sink, &w)) != UP_OK) return st;
  AttnGeometry g;
  if ((st = attn_step_geometry(pb, max_kv_len, w, &g)) != UP_OK) return st;
  *workspace_bytes = g.total;
  return UP_OK;
}

int uniprefill_attention_window_step(const up_params* p, const void* q, const void* k_cache, const void* v_cache,
                                     int64_t v_row_stride, const int32_t* kv_len_dev, int32_t max_kv_len,
                                     const int32_t* block_table, int64_t block_table_stride, int32_t kv_block_size,
                                     int32_t window, int32_t n_sink, void* out, int64_t out_row_stride, float* lse_out,
                                     int64_t lse_row_stride, void* workspace, size_t workspace_bytes, void* stream) {
  Problem pb;
  AttnWindow w;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (pb.T != pb.R || max_kv_len < 0) return UP_ERR_SHAPE;
  if ((st = check_window(window, n_sink, &w)) != UP_OK) return st;
  if (pb.R > 0 && (!q || !out || !kv_len_dev || (max_kv_len > 0 && (!k_cache || !v_cache)))) return UP_ERR_NULL;
  const int e = pb.qk_is_f32 ? 4 : 2;
  if ((st = check_row_stride(v_row_stride, pb.Hkv, pb.head_dim, e)) != UP_OK) return st;
  if ((st = check_row_stride(out_row_stride, pb.Hq, pb.head_dim, e)) != UP_OK) return st;
  if (pb.R > 0 && (st = check_table(block_table, block_table_stride, kv_block_size, max_kv_len)) != UP_OK) return st;
  if (lse_out != nullptr && lse_row_stride < pb.R) return UP_ERR_SHAPE;
  if (pb.k_stride * e > kMaxRowStride || v_row_stride * e > kMaxRowStride) return UP_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out)) return UP_ERR_ALIGN;
  if (!aligned_to(lse_out, 4) || !aligned_to(kv_len_dev, 4)) return UP_ERR_ALIGN;
  AttnGeometry g;
  if ((st = attn_step_geometry(pb, max_kv_len, w, &g)) != UP_OK) return st;
  if (pb.R == 0) return UP_OK;
  if (g.total > 0 && (workspace == nullptr || workspace_bytes < g.total)) return UP_ERR_WORKSPACE;
  if (g.total > 0 && !aligned_to(workspace, 256)) return UP_ERR_ALIGN;
  AttnArgs a{};
  a.q = (const char*)q; a.k = (const char*)k_cache; a.v = (const char*)v_cache; a.out = (char*)out; a.lse = lse_out;
  a.block_table = block_table; a.table_stride = block_table_stride; a.kv_block = kv_block_size;
  a.kv_magic = 0xFFFFFFFFu / (unsigned)kv_block_size;
  a.q_stride_b = pb.q_stride * e; a.k_stride_b = pb.k_stride * e; a.v_stride_b = v_row_stride * e;
  a.out_stride_b = out_row_stride * e; a.lse_stride = lse_row_stride;
  a.c = pb.scale * 1.44269504088896340736f;
  a.R = pb.R; a.Hq = pb.Hq; a.Hkv = pb.Hkv; a.Gq = pb.Gq;
  a.rows = g.rows; a.slots = (int)g.slots; a.items = (int)g.items; a.part_keys = g.part_keys; a.parts = g.parts;
  a.kv_len = kv_len_dev; a.max_len = max_kv_len;
  attn_band_args(g, &w, &a);
  attn_piece_args(g, workspace, &a);
  return launch_attention(a, pb.qk_is_f32, pb.head_dim, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

int uniprefill_linear_attention_plan(const up_params* p, const int32_t* cu_seqlens_host, size_t* workspace_bytes) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (workspace_bytes == nullptr) return UP_ERR_NULL;
  if ((st = check_cu(p, cu_seqlens_host)) != UP_OK) return st;
  LinearGeometry g;
  if ((st = linear_geometry(pb, cu_seqlens_host, &g)) != UP_OK) return st;
  *workspace_bytes = g.total;
  return UP_OK;
}

int uniprefill_linear_attention(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride,
                                const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, const float* log_decay,
                                float* states, int64_t state_stride, int64_t num_states, const int32_t* state_in,
                                const int32_t* state_out, void* out, int64_t out_row_stride, void* workspace,
                                size_t workspace_bytes, void* stream) {
  Problem pb;
  LinearArgs a;
  int st = linear_args(p, q, k, v, v_row_stride, log_decay, states, state_stride, num_states, state_in, state_out, out, out_row_stride, &pb, &a);
  if (st != UP_OK) return st;
  if (!cu_seqlens_dev) return UP_ERR_NULL;
  if ((st = check_cu(p, cu_seqlens_host)) != UP_OK) return st;
  LinearGeometry g;
  if ((st = linear_geometry(pb, cu_seqlens_host, &g)) != UP_OK) return st;
  if (g.total > 0 && (workspace == nullptr || workspace_bytes < g.total)) return UP_ERR_WORKSPACE;
  if (g.total > 0 && !aligned_to(workspace, 256)) return UP_ERR_ALIGN;
  if (pb.R == 0) return UP_OK;
  a.cu = cu_seqlens_dev;
  a.piece = g.piece; a.slots = (int)g.slots;
  if (g.total > 0) a.adds = (float*)workspace;
  return launch_linear(a, pb.qk_is_f32, pb.head_dim, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

int uniprefill_linear_attention_step(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride,
                                     const float* log_decay, float* states, int64_t state_stride, int64_t num_states,
                                     const int32_t* state_in, const int32_t* state_out, void* out, int64_t out_row_stride,
                                     void* stream) {
  Problem pb;
  LinearArgs a;
  int st = linear_args(p, q, k, v, v_row_stride, log_decay, states, state_stride, num_states, state_in, state_out, out, out_row_stride, &pb, &a);
  if (st != UP_OK) return st;
  if (pb.T != pb.R) return UP_ERR_SHAPE;
  if (pb.R == 0) return UP_OK;
  return launch_linear_step(a, pb.qk_is_f32, pb.head_dim, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

int uniprefill_norm_rotate(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride, const void* q_weight,
                           const void* k_weight, float eps, const int32_t* pos, const float* inv_freq, int32_t rot_dim,
                           int32_t pairs, const int32_t* count_dev, void* q_out, int64_t q_out_row_stride, void* k_out,
                           int64_t k_out_row_stride, void* v_out, int64_t v_out_row_stride, const int64_t* slots, int64_t num_slots,
                           void* stream) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (num_slots < 0) return UP_ERR_SHAPE;
  // (eps below the smallest normal float would be taken for 0 by the division)
  if (!(eps >= 0.0f) || isinf(eps) || (eps > 0.0f && eps < 1.17549435e-38f)) return UP_ERR_RANGE;
  if (rot_dim < 0 || rot_dim > pb.head_dim) return UP_ERR_RANGE;
  if (rot_dim % 16 != 0) return UP_ERR_UNSUPPORTED;
  if (eps == 0.0f && (q_weight != nullptr || k_weight != nullptr)) return UP_ERR_RANGE;
  const int e = pb.qk_is_f32 ? 4 : 2;
  if (v != nullptr && (st = check_row_stride(v_row_stride, pb.Hkv, pb.head_dim, e)) != UP_OK) return st;
  if (q_out != nullptr && (st = check_row_stride(q_out_row_stride, pb.Hq, pb.head_dim, e)) != UP_OK) return st;
  if (k_out != nullptr && (st = check_row_stride(k_out_row_stride, pb.Hkv, pb.head_dim, e)) != UP_OK) return st;
  if (v_out != nullptr && (st = check_row_stride(v_out_row_stride, pb.Hkv, pb.head_dim, e)) != UP_OK) return st;
  if (pb.T == 0) return UP_OK;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (v == nullptr) != (v_out == nullptr)) return UP_ERR_NULL;
  if (q == nullptr && k == nullptr && v == nullptr) return UP_ERR_NULL;
  if (rot_dim > 0 && (!pos || !inv_freq)) return UP_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(q_out) || !aligned16(k_out) || !aligned16(v_out)) return UP_ERR_ALIGN;
  if (!aligned16(q_weight) || !aligned16(k_weight) || !aligned_to(pos, 4) || !aligned_to(inv_freq, 4)) return UP_ERR_ALIGN;
  if (!aligned_to(slots, 8) || !aligned_to(count_dev, 4)) return UP_ERR_ALIGN;
  // Rows are turned where they are only if they stay in their places: with another stride, or by slots, a wave would write a row that
  // another one has still to read.
  auto moves = [&](const void* in, int64_t in_stride, const void* out, int64_t out_stride, bool by_slots) {
    return in != nullptr && in == out && (by_slots || in_stride != out_stride);
  };
  if (pb.T > 1 && (moves(q, pb.q_stride, q_out, q_out_row_stride, false) || moves(k, pb.k_stride, k_out, k_out_row_stride, slots != nullptr) ||
                   moves(v, v_row_stride, v_out, v_out_row_stride, slots != nullptr)))
    return UP_ERR_UNSUPPORTED;
  RotateArgs a{};
  a.in[0] = (const char*)q; a.in[1] = (const char*)k; a.in[2] = (const char*)v;
  a.out[0] = (char*)q_out; a.out[1] = (char*)k_out; a.out[2] = (char*)v_out;
  a.in_stride_b[0] = pb.q_stride * e; a.in_stride_b[1] = pb.k_stride * e; a.in_stride_b[2] = v_row_stride * e;
  a.out_stride_b[0] = q_out_row_stride * e; a.out_stride_b[1] = k_out_row_stride * e; a.out_stride_b[2] = v_out_row_stride * e;
  a.weight[0] = (const char*)q_weight; a.weight[1] = (const char*)k_weight;
  a.pos = pos; a.inv_freq = inv_freq; a.slots = slots; a.count_dev = count_dev;
  a.n = pb.T; a.num_slots = num_slots; a.eps = eps;
  a.heads[0] = q != nullptr ? pb.Hq : 0; a.heads[1] = k != nullptr ? pb.Hkv : 0; a.heads[2] = v != nullptr ? pb.Hkv : 0;
  a.D = pb.head_dim; a.rot = rot_dim; a.pairs = pairs != 0;
  // A wave takes a token's heads in rounds of 2048 bytes; where the tokens are few, several waves share a token.
  const int64_t rounds = (((int64_t)a.heads[0] + a.heads[1] + a.heads[2]) * a.D * e + 2047) / 2048;
  int64_t waves = (8 * kCUs + pb.T - 1) / pb.T;
  waves = waves < rounds ? waves : rounds;
  if (waves * pb.T > (int64_t)UINT32_MAX / 64 - 256) return UP_ERR_UNSUPPORTED;
  a.waves = (int)waves;
  // (past the cache: 32768 tokens of 40/8 heads, 940 MB, 208 -> 197 us; what fits stays for the layer that reads it: 2000 tokens of 32/8
  // heads, 49 MB, would go from 12.0 to 13.7 us and be gone from the cache)
  a.stream = 2 * rounds * 2048 * pb.T > (int64_t)256 << 20;
  return launch_rotate(a, pb.qk_is_f32, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

int uniprefill_append_pages(const int32_t* kv_len_dev, const int32_t* num_new_dev, int32_t num_seqs, int32_t kv_block_size,
                            int32_t* block_table, int64_t block_table_stride, const int32_t* free_pages,
                            const int32_t* num_free_dev, int32_t* free_left_dev, int32_t* new_len_dev, int32_t* cu_seqlens_dev,
                            int32_t* cu_seqlens_k_dev, int32_t* pos, int64_t* slots, int64_t capacity, int32_t* num_served_dev,
                            void* stream) {
  return append_pages_impl(kv_len_dev, num_new_dev, nullptr, num_seqs, kv_block_size, block_table, block_table_stride, free_pages, num_free_dev,
                           free_left_dev, new_len_dev, cu_seqlens_dev, cu_seqlens_k_dev, pos, slots, capacity, num_served_dev, stream);
}

int uniprefill_append_pages_dropped(const int32_t* kv_len_dev, const int32_t* num_new_dev, const int32_t* num_dropped_dev, int32_t num_seqs, int32_t kv_block_size,
                                    int32_t* block_table, int64_t block_table_stride, const int32_t* free_pages, const int32_t* num_free_dev,
                                    int32_t* free_left_dev, int32_t* new_len_dev, int32_t* cu_seqlens_dev, int32_t* cu_seqlens_k_dev, int32_t* pos,
                                    int64_t* slots, int64_t capacity, int32_t* num_served_dev, void* stream) {
  return append_pages_impl(kv_len_dev, num_new_dev, num_dropped_dev, num_seqs, kv_block_size, block_table, block_table_stride, free_pages, num_free_dev,
                           free_left_dev, new_len_dev, cu_seqlens_dev, cu_seqlens_k_dev, pos, slots, capacity, num_served_dev, stream);
}

}  // extern "C"
