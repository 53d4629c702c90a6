// Entry points of the attention layer's operators (attention of a packed batch, the 4-bit KV cache,
// eviction): argument checks and launch geometry, host code only.  Part of up_api.hip, whose checks
// of the common arguments it uses.
#pragma once

#include "up_attn.h"

namespace {

// bytes between key (value) rows up to which a work-group's offsets of a few rows stay within 32 bits
constexpr int64_t kMaxRowStride = 1 << 27;
// tokens of a sequence up to which the kernels may count some tiles past its end
constexpr int kMaxLength = INT32_MAX - 65536;

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// ---- attention of a packed batch
// The geometry follows from the host's lengths: a captured call keeps those it was made with.
// A work-group takes 256 rows (tokens x query heads of one kv head; 8 waves) of one sequence and walks over the
// keys they see; 128 rows (4 waves) where work-groups of 256 would be fewer than the CUs, or fewer than twice as many with the
// longest well beyond a CU's share (one prompt of 2048, 32/8 heads, 67 -> 57 us, float 500 -> 296; 2048 tokens after 6000 others
// are even and stay: 244 us, 254 in work-groups of 128).  Where the rows alone leave
// the chip idle all the same -- decode rows and short chunks on long caches -- the keys of every row tile are cut into
// pieces of part_keys and the pieces joined.
struct AttnWindow {
  int window, n_sink;
};
struct AttnGeometry {
  int rows;
  int sinks;                 // windowed attention: the sinks in whole stages
  int reach;                 // ... and the keys that a row tile walks over at most
  int part_keys, parts;      // 0, 1: not cut
  long long items;           // work-groups per kv head
  long long pieces;          // row tiles x pieces of the sequences that are cut
  long long slots;           // row tiles in the numbering that needs no prefix sums
  size_t base_off, o_off, ml_off, total;
};

// What a cut gains and costs, in microseconds.  A CU works through the keys of 128 rows at key_us each; with the keys cut into
// pieces of half a CU's share, not the longest tile decides but the share and one piece more.  Every piece then leaves float rows that are
// written and read back (3 TB/s) by one more launch.
// key_us is measured (one tile on a CU of its own); batches on both sides of the rule, not cut -> cut: one token after 8191, 56 -> 28 us
// (in pieces of 2048 and of 512 keys); 1000 tokens float, 8/8 heads, 137 -> 57; 2048 tokens, 32/8 heads, 67 -> 98 (not cut);
// 1000 tokens, 32/8 heads, 28 -> 39 (not cut).  Pieces shorter than 512 keys (256 float) cost more to join than they save.
double attn_key_us(bool f32, int D) { return f32 ? (D == 64 ? 0.06 : 0.13) : D == 64 ? 0.01 : D == 128 ? 0.015 : 0.04; }

// Keys that a tile of `rows` rows walks over at most: the sinks in whole stages, and the windows of its tokens, which begin up to 7 keys early.
long long attn_window_reach(const Problem& pb, const AttnWindow& w, int rows, int* sinks) {
  const long long unit = attn_stage_keys(pb.head_dim * (pb.qk_is_f32 ? 4 : 2), rows), whole = (w.n_sink + unit - 1) / unit * unit;
  // (as many sinks as no sequence has tokens: the band begins among them everywhere)
  *sinks = whole > kMaxLength ? kMaxLength : (int)whole;
  return *sinks + (long long)w.window + rows / pb.Gq + 2 + 7;
}

int attn_geometry(const Problem& pb, const int32_t* cu, const int32_t* ck, AttnGeometry* g, const AttnWindow* w = nullptr) {
  const int D = pb.head_dim;
  *g = AttnGeometry{};
  g->rows = 256;
  long long longest = 0, live = 0;
  for (int r = 0; r < pb.R; ++r) {
    const long long N = cu[r + 1] - cu[r], L = ck[r + 1] - ck[r];
    live += (N * pb.Gq + 255) / 256;
    if (N > 0) longest = L > longest ? L : longest;
  }
  if (longest > kMaxLength) return UP_ERR_UNSUPPORTED;
  auto tiles_of = [&](long long N, int rows) { return (N * pb.Gq + rows - 1) / rows; };
  auto reach_of = [&](int rows) { return w != nullptr ? attn_window_reach(pb, *w, rows, &g->sinks) : (long long)INT32_MAX; };
  longest = longest < reach_of(128) ? longest : reach_of(128);
  auto keys_per_cu = [&](int rows) {
    double work = 0;
    for (int r = 0; r < pb.R; ++r) {
      const long long N = cu[r + 1] - cu[r], L = ck[r + 1] - ck[r], tiles = tiles_of(N, rows);
      const double all = (double)tiles * (double)(L - N) + 0.5 * (double)(tiles + 1) * (double)N, most = (double)tiles * (double)reach_of(rows);
      if (N > 0) work += all < most ? all : most;
    }
    return work * pb.Hkv / kCUs;
  };
  if (live * pb.Hkv < kCUs || (live * pb.Hkv < 2 * kCUs && 2.0 * (double)longest > 1.5 * keys_per_cu(128))) g->rows = 128;
  // (work-items of a launch are counted in 32 bits, and one of more runs short without an error; twice as many work-groups
  // of 128 rows fit as of 256)
  auto most_groups = [](int threads) { return (long long)UINT32_MAX / threads; };
  if (((long long)pb.T * pb.Gq / 256 + pb.R) * pb.Hkv > most_groups(2 * 256)) g->rows = 128;
  // Narrow windows: 128 rows walk over fewer keys that some of them do not see (32768 tokens, 32/8 heads of 128, window 512, 499 -> 450 us;
  // 64 wide, window 1000, 430 -> 408; window 4096 1968 -> 2025; 256 wide, where 128 rows leave a CU four waves, 341 -> 473)
  if (w != nullptr && D * (pb.qk_is_f32 ? 4 : 2) < 512 && reach_of(256) <= 2048) g->rows = 128;
  const double fair = keys_per_cu(g->rows);
  const long long reach = reach_of(g->rows);
  g->reach = reach < INT32_MAX ? (int)reach : INT32_MAX;
  auto pieces_of = [&](int r, long long part) { return attn_pieces(imin(ck[r + 1] - ck[r], g->reach), (int)part); };
  g->parts = 1;
  g->slots = (long long)pb.T * pb.Gq / g->rows + pb.R;
  g->items = g->slots;
  const long long fewest = pb.qk_is_f32 ? 256 : 512;
  if ((double)longest > fair && longest > fewest) {
    const long long want = fair > 2.0 * (double)fewest ? (long long)(0.5 * fair) : fewest;
    const long long part = (want + 127) / 128 * 128;
    double rows = 0;      // rows of float sums that the pieces leave
    for (int r = 0; r < pb.R; ++r) {
      const long long N = cu[r + 1] - cu[r], n = pieces_of(r, part);
      if (n > 1) rows += (double)(N * pb.Hq) * (double)n;
    }
    const double gain = ((double)longest - fair - (double)part) * attn_key_us(pb.qk_is_f32, D) * g->rows / 128, cost = 6.0 + rows * D * 8.0 / 3e6;
    if (part < longest && gain > cost) {
      g->part_keys = (int)part;
      g->parts = attn_pieces((int)longest, (int)part);
      g->items = 0;
      for (int r = 0; r < pb.R; ++r) {
        const long long tiles = tiles_of(cu[r + 1] - cu[r], g->rows), n = pieces_of(r, part);
        g->items += tiles * n;
        if (n > 1) g->pieces += tiles * n;
      }
      size_t off = 0;
      g->base_off = off;
      off = align256(off + (size_t)g->slots * sizeof(int32_t));
      g->o_off = off;
      off = align256(off + (size_t)g->pieces * pb.Hkv * g->rows * D * sizeof(float));
      g->ml_off = off;
      off = align256(off + (size_t)g->pieces * pb.Hkv * g->rows * 2 * sizeof(float));
      g->total = off;
    }
  }
  if (g->items * pb.Hkv > most_groups(2 * g->rows) || g->slots * pb.Hkv > most_groups(256)) return UP_ERR_UNSUPPORTED;
  return UP_OK;
}

// One new token per sequence, lengths on the device: the keys that it can see at most are cut into pieces for about two work-groups per CU.
int attn_step_geometry(const Problem& pb, int max_len, const AttnWindow& w, AttnGeometry* g) {
  *g = AttnGeometry{};
  if (max_len > kMaxLength) return UP_ERR_UNSUPPORTED;
  g->rows = 128;
  const long long reach = attn_window_reach(pb, w, g->rows, &g->sinks);
  g->reach = (int)(reach < max_len ? reach : max_len);
  const long long groups = (long long)pb.R * pb.Hkv, want = groups > 0 ? (2 * kCUs + groups - 1) / groups : 1;
  long long part = ((g->reach + want - 1) / want + 127) / 128 * 128;
  if (part < 128) part = 128;
  g->parts = imax(1, attn_pieces(g->reach, (int)part));
  g->slots = pb.R;
  g->items = (long long)pb.R * g->parts;
  if (g->parts > 1) {
    g->part_keys = (int)part;
    g->pieces = g->items;
    size_t off = align256((size_t)g->slots * sizeof(int32_t));
    g->o_off = off;
    off = align256(off + (size_t)g->pieces * pb.Hkv * g->rows * pb.head_dim * sizeof(float));
    g->ml_off = off;
    off = align256(off + (size_t)g->pieces * pb.Hkv * g->rows * 2 * sizeof(float));
    g->total = off;
  }
  if (g->items * pb.Hkv > (long long)UINT32_MAX / 512) return UP_ERR_UNSUPPORTED;
  return UP_OK;
}

// strides of a second tensor with head rows (values, outputs), in elements
int check_row_stride(int64_t stride, int heads, int head_dim, int elem) {
  if (stride < (int64_t)heads * head_dim) return UP_ERR_SHAPE;
  if (stride > kMostStride) return UP_ERR_UNSUPPORTED;
  if ((stride * elem) % 16 != 0) return UP_ERR_ALIGN;
  return UP_OK;
}

bool aligned_to(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1u)) == 0; }

void attn_band_args(const AttnGeometry& g, const AttnWindow* w, AttnArgs* a) {
  if (w == nullptr) return;
  a->window = w->window; a->n_sink = w->n_sink; a->sinks = g.sinks; a->reach = g.reach;
}
void attn_piece_args(const AttnGeometry& g, void* workspace, AttnArgs* a) {
  if (g.part_keys == 0) return;
  a->base = (int32_t*)((char*)workspace + g.base_off);
  a->o_part = (float*)((char*)workspace + g.o_off);
  a->ml_part = (float*)((char*)workspace + g.ml_off);
}

int attention_plan_impl(const up_params* p, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k_host, const AttnWindow* w,
                        size_t* workspace_bytes) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (workspace_bytes == nullptr) return UP_ERR_NULL;
  if ((st = check_cu(p, cu_seqlens_host)) != UP_OK) return st;
  if (cu_seqlens_k_host != nullptr && (st = check_cu_k(p, cu_seqlens_host, cu_seqlens_k_host)) != UP_OK) return st;
  AttnGeometry g;
  if ((st = attn_geometry(pb, cu_seqlens_host, cu_seqlens_k_host != nullptr ? cu_seqlens_k_host : cu_seqlens_host, &g,
                          w)) != UP_OK)
    return st;
  *workspace_bytes = g.total;
  return UP_OK;
}

int attention_impl(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride,
                   const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k_dev,
                   const int32_t* cu_seqlens_k_host, const PagedKeys& paged, const AttnWindow* w, void* out, int64_t out_row_stride,
                   float* lse_out, int64_t lse_row_stride, void* workspace, size_t workspace_bytes, void* stream) {
  KeySide ks;
  int st = optional_key_side(cu_seqlens_k_dev, cu_seqlens_k_host, &paged, &ks);
  if (st != UP_OK) return st;
  Problem pb;
  if ((st = check_params(p, true, false, &pb)) != UP_OK) return st;
  if (!cu_seqlens_dev || (pb.T > 0 && (!q || !k || !v || !out))) return UP_ERR_NULL;
  if ((st = check_cu(p, cu_seqlens_host)) != UP_OK) return st;
  if ((st = check_key_side(p, cu_seqlens_host, ks)) != UP_OK) return st;
  const int e = pb.qk_is_f32 ? 4 : 2;
  if ((st = check_row_stride(v_row_stride, pb.Hkv, pb.head_dim, e)) != UP_OK) return st;
  if ((st = check_row_stride(out_row_stride, pb.Hq, pb.head_dim, e)) != UP_OK) return st;
  if (lse_out != nullptr && lse_row_stride < pb.T) return UP_ERR_SHAPE;
  if (pb.k_stride * e > kMaxRowStride || v_row_stride * e > kMaxRowStride) return UP_ERR_UNSUPPORTED;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return UP_ERR_ALIGN;
  if (!aligned_to(lse_out, 4) || !aligned_to(paged.block_table, 4)) return UP_ERR_ALIGN;
  const int32_t* ck = ks.ctx ? cu_seqlens_k_host : cu_seqlens_host;
  AttnGeometry g;
  if ((st = attn_geometry(pb, cu_seqlens_host, ck, &g, w)) != UP_OK) return st;
  if (g.total > 0 && (workspace == nullptr || workspace_bytes < g.total)) return UP_ERR_WORKSPACE;
  if (g.total > 0 && !aligned_to(workspace, 256)) return UP_ERR_ALIGN;
  if (pb.T == 0) return UP_OK;
  AttnArgs a{};
  a.q = (const char*)q; a.k = (const char*)k; a.v = (const char*)v; a.out = (char*)out; a.lse = lse_out;
  a.cu = cu_seqlens_dev; a.cu_k = ks.ctx ? cu_seqlens_k_dev : cu_seqlens_dev;
  if (ks.paged != nullptr) {
    a.block_table = paged.block_table; a.table_stride = paged.table_stride; a.kv_block = paged.kv_block;
    a.kv_magic = 0xFFFFFFFFu / (unsigned)paged.kv_block;
  }
  a.q_stride_b = pb.q_stride * e; a.k_stride_b = pb.k_stride * e; a.v_stride_b = v_row_stride * e;
  a.out_stride_b = out_row_stride * e; a.lse_stride = lse_row_stride;
  a.c = pb.scale * 1.44269504088896340736f;
  a.R = pb.R; a.Hq = pb.Hq; a.Hkv = pb.Hkv; a.Gq = pb.Gq;
  a.rows = g.rows; a.slots = (int)g.slots; a.items = (int)g.items; a.part_keys = g.part_keys; a.parts = g.parts;
  attn_band_args(g, w, &a);
  attn_piece_args(g, workspace, &a);
  return launch_attention(a, pb.qk_is_f32, pb.head_dim, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

// ---- the 4-bit cache
int check_q4_cache(const Problem& pb, const void* k_cache, const void* v_cache, int64_t cache_row_stride) {
  if (cache_row_stride < q4_row_bytes(pb.Hkv, pb.head_dim)) return UP_ERR_SHAPE;
  if (cache_row_stride % 16 != 0 || !aligned16(k_cache) || !aligned16(v_cache)) return UP_ERR_ALIGN;
  return UP_OK;
}

int q4_copy_impl(bool store, const up_params* p, const void* k, const void* v, int64_t v_row_stride, void* k_cache,
                 void* v_cache, int64_t cache_row_stride, int64_t num_slots, const int64_t* slots, int64_t n,
                 const int32_t* count_dev, void* stream) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (n < 0 || num_slots < 0) return UP_ERR_SHAPE;
  const int e = pb.qk_is_f32 ? 4 : 2;
  if ((st = check_row_stride(v_row_stride, pb.Hkv, pb.head_dim, e)) != UP_OK) return st;
  if ((st = check_q4_cache(pb, k_cache, v_cache, cache_row_stride)) != UP_OK) return st;
  if (n == 0) return UP_OK;
  if ((k == nullptr) != (k_cache == nullptr) || (v == nullptr) != (v_cache == nullptr)) return UP_ERR_NULL;
  if ((k == nullptr && v == nullptr) || slots == nullptr) return UP_ERR_NULL;
  if (!aligned16(k) || !aligned16(v) || !aligned_to(slots, 8) || !aligned_to(count_dev, 4)) return UP_ERR_ALIGN;
  if (n > (INT32_MAX - 256) / ((int64_t)pb.Hkv * (pb.head_dim / kQ4Group))) return UP_ERR_UNSUPPORTED;      // groups of 64 elements
  Q4CopyArgs a{};
  a.rows_in[0] = (const char*)k; a.rows_in[1] = (const char*)v;
  a.rows_out[0] = (char*)const_cast<void*>(k); a.rows_out[1] = (char*)const_cast<void*>(v);
  a.cache[0] = (char*)k_cache; a.cache[1] = (char*)v_cache;
  a.row_stride_b[0] = pb.k_stride * e; a.row_stride_b[1] = v_row_stride * e;
  a.cache_stride = cache_row_stride; a.slots = slots; a.count_dev = count_dev; a.n = n; a.num_slots = num_slots;
  a.heads = pb.Hkv; a.D = pb.head_dim;
  const hipError_t err = store ? launch_q4_store(a, pb.qk_is_f32, (hipStream_t)stream) : launch_q4_load(a, pb.qk_is_f32, (hipStream_t)stream);
  return err == hipSuccess ? UP_OK : UP_ERR_HIP;
}

// Decode: a work-group has eight waves (four at D = 256), each on a kv head of its own; with fewer heads than
// waves the ones that are left share the keys of the work-group (wave_parts of them per head).  The lengths are known on the
// device alone: the host sizes the launch to what the chip holds at once (fewer if max_kv_len leaves less to do), and the
// kernel cuts the steps of all sequences evenly among its work-groups.
struct Q4Geometry {
  int groups, wave_parts, head_groups;
  long long logit_stride;
  size_t step_off, o_off, ml_off, lse2_off, logit_off, total;
};

int q4_geometry(const Problem& pb, int max_len, bool mass, Q4Geometry* g) {
  *g = Q4Geometry{};
  g->wave_parts = 1;
  const int waves = q4_waves(pb.head_dim);
  // (as many as there are waves, and rows in LDS: 18 pieces of 16 bytes a key at D = 64, 36 beyond)
  const long long row_places = pb.Hkv * (pb.head_dim / 32) + (pb.Hkv * (pb.head_dim / kQ4Group) * 4 + 15) / 16;
  while (g->wave_parts < kQ4MaxWaveParts && (g->wave_parts + 1) * pb.Hkv <= waves &&
         (g->wave_parts + 1) * row_places <= (pb.head_dim == 64 ? 18 : 36))
    ++g->wave_parts;
  g->head_groups = (pb.Hkv + waves - 1) / waves;
  const int layers = g->head_groups * ((pb.Gq + 15) / 16), places = kCUs * (pb.head_dim == 64 ? 2 : 1);
  const long long steps = (long long)pb.R * ((max_len + 64ll * g->wave_parts - 1) / (64ll * g->wave_parts));
  long long groups = places / layers;
  groups = groups < 1 ? 1 : groups;
  groups = groups < steps ? groups : steps;
  g->groups = groups < 1 ? 1 : (int)groups;
  const size_t rows = (size_t)pb.R * pb.Hq, pieces = ((size_t)g->groups + pb.R) * g->wave_parts * pb.Hq;
  size_t off = 0;
  g->step_off = off;
  off = align256(off + ((size_t)pb.R + 1) * sizeof(unsigned));
  g->o_off = off;
  off = align256(off + pieces * pb.head_dim * sizeof(float));
  g->ml_off = off;
  off = align256(off + pieces * 2 * sizeof(float));
  if (mass) {
    g->logit_stride = ((long long)max_len + 63) / 64 * 64;
    g->lse2_off = off;
    off = align256(off + rows * sizeof(float));
    g->logit_off = off;
    off = align256(off + rows * (size_t)g->logit_stride * sizeof(float));
  }
  g->total = off;
  if (pb.R > 65535 || layers > 65535 || steps > INT32_MAX || max_len > kMaxLength || pb.Hq > UINT32_MAX / (64 * kQ4JoinWaves))
    return UP_ERR_UNSUPPORTED;
  return UP_OK;
}

int check_table(const void* table, int64_t stride, int32_t block, long long tokens) {
  if (block < 1 || stride < 0) return UP_ERR_RANGE;
  if (tokens > 0 && table == nullptr) return UP_ERR_NULL;
  if (!aligned_to(table, 4)) return UP_ERR_ALIGN;
  if ((tokens + block - 1) / block > stride) return UP_ERR_SHAPE;
  return UP_OK;
}

}  // namespace

extern "C" {

int uniprefill_attention_plan(const up_params* p, const int32_t* cu_seqlens_host, const int32_t* cu_seqlens_k_host,
                              size_t* workspace_bytes) {
  return attention_plan_impl(p, cu_seqlens_host, cu_seqlens_k_host, nullptr, workspace_bytes);
}

int uniprefill_attention(const up_params* p, const void* q, const void* k, const void* v, int64_t v_row_stride,
                         const int32_t* cu_seqlens_dev, const int32_t* cu_seqlens_host,
                         const int32_t* cu_seqlens_k_dev, const int32_t* cu_seqlens_k_host,
                         const int32_t* block_table, int64_t block_table_stride, int32_t kv_block_size, void* out,
                         int64_t out_row_stride, float* lse_out, int64_t lse_row_stride, void* workspace,
                         size_t workspace_bytes, void* stream) {
  return attention_impl(p, q, k, v, v_row_stride, cu_seqlens_dev, cu_seqlens_host, cu_seqlens_k_dev, cu_seqlens_k_host,
                        PagedKeys{block_table, block_table_stride, kv_block_size}, nullptr, out, out_row_stride, lse_out, lse_row_stride,
                        workspace, workspace_bytes, stream);
}

int64_t uniprefill_q4_row_bytes(int32_t num_kv_heads, int32_t head_dim) {
  if (num_kv_heads < 1 || (head_dim != 64 && head_dim != 128 && head_dim != 256)) return 0;
  return q4_row_bytes(num_kv_heads, head_dim);
}

int uniprefill_cache_store_q4(const up_params* p, const void* k, const void* v, int64_t v_row_stride,
                              const int64_t* slots, int64_t n, const int32_t* count_dev, void* k_cache, void* v_cache,
                              int64_t cache_row_stride, int64_t num_slots, void* stream) {
  return q4_copy_impl(true, p, k, v, v_row_stride, k_cache, v_cache, cache_row_stride, num_slots, slots, n, count_dev, stream);
}

int uniprefill_cache_load_q4(const up_params* p, const void* k_cache, const void* v_cache, int64_t cache_row_stride,
                             int64_t num_slots, const int64_t* slots, int64_t n, const int32_t* count_dev, void* k_out,
                             void* v_out, int64_t v_row_stride, void* stream) {
  return q4_copy_impl(false, p, k_out, v_out, v_row_stride, const_cast<void*>(k_cache), const_cast<void*>(v_cache),
                      cache_row_stride, num_slots, slots, n, count_dev, stream);
}

int uniprefill_attention_q4_plan(const up_params* p, int32_t max_kv_len, int32_t want_mass, size_t* workspace_bytes) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (workspace_bytes == nullptr) return UP_ERR_NULL;
  if (pb.qk_is_f32) return UP_ERR_UNSUPPORTED;
  if (pb.T != pb.R || max_kv_len < 0) return UP_ERR_SHAPE;
  Q4Geometry g;
  if ((st = q4_geometry(pb, max_kv_len, want_mass != 0, &g)) != UP_OK) return st;
  *workspace_bytes = g.total;
  return UP_OK;
}

int uniprefill_attention_q4(const up_params* p, const void* q, const void* k_cache, const void* v_cache,
                            int64_t cache_row_stride, const int32_t* kv_len_dev, int32_t max_kv_len,
                            const int32_t* block_table, int64_t block_table_stride, int32_t kv_block_size, void* out,
                            int64_t out_row_stride, float* lse_out, int64_t lse_row_stride, const float* mass_in,
                            float* mass_out, int64_t mass_row_stride, void* workspace, size_t workspace_bytes,
                            void* stream) {
  Problem pb;
  int st = check_params(p, true, false, &pb);
  if (st != UP_OK) return st;
  if (pb.qk_is_f32) return UP_ERR_UNSUPPORTED;
  if (pb.T != pb.R || max_kv_len < 0) return UP_ERR_SHAPE;
  if (pb.R > 0 && (!q || !out || !kv_len_dev || (max_kv_len > 0 && (!k_cache || !v_cache)))) return UP_ERR_NULL;
  if (mass_in != nullptr && mass_out == nullptr) return UP_ERR_NULL;
  if ((st = check_q4_cache(pb, k_cache, v_cache, cache_row_stride)) != UP_OK) return st;
  if ((st = check_row_stride(out_row_stride, pb.Hq, pb.head_dim, 2)) != UP_OK) return st;
  if (pb.R > 0 && (st = check_table(block_table, block_table_stride, kv_block_size, max_kv_len)) != UP_OK) return st;
  if (lse_out != nullptr && lse_row_stride < pb.R) return UP_ERR_SHAPE;
  if (mass_out != nullptr && mass_row_stride < max_kv_len) return UP_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(out)) return UP_ERR_ALIGN;
  if (!aligned_to(lse_out, 4) || !aligned_to(mass_in, 4) || !aligned_to(mass_out, 4) || !aligned_to(kv_len_dev, 4)) return UP_ERR_ALIGN;
  Q4Geometry g;
  if ((st = q4_geometry(pb, max_kv_len, mass_out != nullptr, &g)) != UP_OK) return st;
  if (pb.R == 0) return UP_OK;
  if (g.total > 0 && (workspace == nullptr || workspace_bytes < g.total)) return UP_ERR_WORKSPACE;
  if (g.total > 0 && !aligned_to(workspace, 256)) return UP_ERR_ALIGN;
  Q4AttnArgs a{};
  a.q = (const char*)q; a.k = (const char*)k_cache; a.v = (const char*)v_cache; a.out = (char*)out; a.lse = lse_out;
  a.kv_len = kv_len_dev; a.block_table = block_table; a.table_stride = block_table_stride;
  a.cache_stride = cache_row_stride; a.q_stride_b = pb.q_stride * 2; a.out_stride_b = out_row_stride * 2;
  a.lse_stride = lse_row_stride; a.mass_in = mass_in; a.mass_out = mass_out; a.mass_stride = mass_row_stride;
  a.kv_block = kv_block_size; a.kv_magic = 0xFFFFFFFFu / (unsigned)kv_block_size;
  a.c = pb.scale * 1.44269504088896340736f;
  a.R = pb.R; a.Hq = pb.Hq; a.Hkv = pb.Hkv; a.Gq = pb.Gq; a.D = pb.head_dim; a.max_len = max_kv_len;
  a.groups = g.groups; a.wave_parts = g.wave_parts; a.head_groups = g.head_groups;
  char* ws = (char*)workspace;
  a.seq_step = (unsigned*)(ws + g.step_off);
  a.o_part = (float*)(ws + g.o_off);
  a.ml_part = (float*)(ws + g.ml_off);
  if (mass_out != nullptr) {
    a.lse2 = (float*)(ws + g.lse2_off);
    a.logits = (float*)(ws + g.logit_off);
    a.logit_stride = g.logit_stride;
  }
  return launch_q4_attention(a, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

int uniprefill_cache_evict(void* k_cache, void* v_cache, int64_t row_bytes, int64_t cache_row_stride, const float* mass,
                           int64_t mass_row_stride, const int32_t* kv_len_dev, int32_t num_seqs, int32_t max_kv_len,
                           int32_t budget, int32_t n_sink, int32_t n_recent, const int32_t* block_table,
                           int64_t block_table_stride, const int32_t* new_table, int64_t new_table_stride,
                           int32_t kv_block_size, int32_t* kept_idx, float* mass_out, int64_t mass_out_stride,
                           int32_t* new_len, void* stream) {
  if (num_seqs < 0 || max_kv_len < 0) return UP_ERR_SHAPE;
  if (n_sink < 0 || n_recent < 0 || budget < 1 || (int64_t)n_sink + n_recent > budget) return UP_ERR_RANGE;
  if (row_bytes < 16 || row_bytes > cache_row_stride) return UP_ERR_SHAPE;
  if (mass_row_stride < max_kv_len || mass_out_stride < budget) return UP_ERR_SHAPE;
  if (row_bytes % 16 != 0 || cache_row_stride % 16 != 0 || !aligned16(k_cache) || !aligned16(v_cache)) return UP_ERR_ALIGN;
  if (num_seqs == 0) return UP_OK;
  if (!kv_len_dev || !new_len) return UP_ERR_NULL;
  if (max_kv_len > 0 && (!k_cache || !mass || !kept_idx || !mass_out)) return UP_ERR_NULL;
  int st = check_table(block_table, block_table_stride, kv_block_size, max_kv_len);
  if (st != UP_OK) return st;
  const int most = budget < max_kv_len ? budget : max_kv_len;      // tokens that a sequence can keep
  if ((st = check_table(new_table, new_table_stride, kv_block_size, most)) != UP_OK) return st;
  if (!aligned_to(mass, 4) || !aligned_to(mass_out, 4) || !aligned_to(kept_idx, 4) || !aligned_to(kv_len_dev, 4) || !aligned_to(new_len, 4))
    return UP_ERR_ALIGN;
  // (the kernels count 16-byte pieces in 31 bits, those of one row too where max_kv_len leaves no rows)
  if (num_seqs > 65535 || max_kv_len > kMaxLength || imax(most, 1) > (INT32_MAX - 1024) / (row_bytes / 16)) return UP_ERR_UNSUPPORTED;
  if (max_kv_len > 0 && ((const void*)mass == mass_out || (const void*)kept_idx == mass_out || (const void*)mass == kept_idx)) return UP_ERR_UNSUPPORTED;
  // the lengths are read by the last launch too, which writes them: in place, or apart
  const intptr_t apart = (intptr_t)new_len - (intptr_t)kv_len_dev, ends = (intptr_t)num_seqs * (intptr_t)sizeof(int32_t);
  if (apart != 0 && apart > -ends && apart < ends) return UP_ERR_UNSUPPORTED;
  EvictArgs a{};
  a.k = (char*)k_cache; a.v = (char*)v_cache; a.row_bytes = row_bytes; a.cache_stride = cache_row_stride;
  a.mass = mass; a.mass_out = mass_out; a.mass_stride = mass_row_stride; a.mass_out_stride = mass_out_stride;
  a.kv_len = kv_len_dev; a.block_table = block_table; a.new_table = new_table; a.table_stride = block_table_stride;
  a.new_table_stride = new_table_stride; a.kept_idx = kept_idx; a.new_len = new_len;
  a.R = num_seqs; a.max_len = max_kv_len; a.budget = budget; a.n_sink = n_sink; a.n_recent = n_recent;
  a.kv_block = kv_block_size; a.kv_magic = 0xFFFFFFFFu / (unsigned)kv_block_size;
  a.piece_magic = 0xFFFFFFFFu / (unsigned)(row_bytes / 16);
  return launch_evict(a, (hipStream_t)stream) == hipSuccess ? UP_OK : UP_ERR_HIP;
}

}  // extern "C"

#include "up_layers_api.h"
