// Host side of the paged cache, shared by its C entry points: argument checks,
// workspace sections and launch planning.
#pragma once

#include <math.h>
#include <string.h>

#include <algorithm>

#include "paged.h"

namespace glide {
namespace {

constexpr int32_t kMaxPagedWindow = 1 << 30;
constexpr int32_t kMaxSinks = 1 << 20;
constexpr int64_t kMaxUnits = int64_t(1) << 20;       // B * Hkv, a grid dimension
constexpr int64_t kMaxLaunchRows = int64_t(1) << 27;  // rows of one prefill launch
// Workgroups of one launch, where a row may be one: a grid has fewer than 2^32 threads.
constexpr int64_t kMaxLaunchUnits = int64_t(1) << 23;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int esize(const glide_paged_config* c) { return c->dtype == GLIDE_BF16 ? 2 : 4; }

glide_status check_cfg(const glide_paged_config* c) {
  if (!c) return GLIDE_ERR_NULL;
  if (c->batch < 1 || c->batch > (1 << 20)) return GLIDE_ERR_INVALID;
  if (c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads > 4096) return GLIDE_ERR_INVALID;
  if (c->n_q_heads % c->n_kv_heads) return GLIDE_ERR_INVALID;
  if (c->head_dim < 1) return GLIDE_ERR_INVALID;
  if (c->dtype != GLIDE_F32 && c->dtype != GLIDE_BF16) return GLIDE_ERR_INVALID;
  if (c->page_size < 1 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) return GLIDE_ERR_INVALID;
  if (c->n_pages < 1 || c->max_pages < 1) return GLIDE_ERR_INVALID;
  if (int64_t(c->max_pages) * c->page_size > kMaxPagedWindow) return GLIDE_ERR_INVALID;
  if (c->window < 0 || c->window > kMaxPagedWindow) return GLIDE_ERR_INVALID;
  if (c->n_sinks < 0 || c->n_sinks > kMaxSinks) return GLIDE_ERR_INVALID;
  if (c->window == 0 && c->n_sinks == 0) return GLIDE_ERR_INVALID;
  if (!isfinite(c->sm_scale)) return GLIDE_ERR_INVALID;
  if (c->n_q_heads / c->n_kv_heads > kMaxG) return GLIDE_ERR_UNSUPPORTED;
  if (c->head_dim != 64 && c->head_dim != 128) return GLIDE_ERR_UNSUPPORTED;
  if (int64_t(c->batch) * c->n_kv_heads > kMaxUnits) return GLIDE_ERR_UNSUPPORTED;
  return GLIDE_OK;
}

glide_status check_cache(const glide_paged_config* c, const glide_paged_cache* k) {
  if (!k || !k->k || !k->v || !k->block_table || !k->lens) return GLIDE_ERR_NULL;
  if (!aligned(k->k, 16) || !aligned(k->v, 16) || !aligned(k->weights, 4) || !aligned(k->block_table, 4) ||
      !aligned(k->lens, 4))
    return GLIDE_ERR_ALIGN;
  for (int i = 0; i < 3; ++i) {
    const int64_t most = (int64_t(1) << 46) / esize(c);  // no product of a stride and an index overflows
    if (k->k_strides[i] < 0 || k->v_strides[i] < 0 || k->k_strides[i] > most || k->v_strides[i] > most)
      return GLIDE_ERR_INVALID;
    if (k->k_strides[i] * esize(c) % 16 || k->v_strides[i] * esize(c) % 16) return GLIDE_ERR_ALIGN;
  }
  return GLIDE_OK;
}

glide_status check_cache4(const glide_paged_config* c, const glide_nibble_cache* k) {
  if (!k || !k->k_codes || !k->k_scales || !k->v_codes || !k->v_scales || !k->block_table || !k->lens)
    return GLIDE_ERR_NULL;
  if (!aligned(k->k_codes, 16) || !aligned(k->v_codes, 16) || !aligned(k->k_scales, 16) || !aligned(k->v_scales, 16) ||
      !aligned(k->block_table, 4) || !aligned(k->lens, 4))
    return GLIDE_ERR_ALIGN;
  // the kernels number the pools' rows in 32 bits
  if (int64_t(c->n_pages) * c->n_kv_heads > (int64_t(1) << 32) / c->page_size) return GLIDE_ERR_UNSUPPORTED;
  return GLIDE_OK;
}

// cu_seqlens of a call over new tokens; one sequence's rows of q span less than
// 2 GiB.
glide_status check_cu(const glide_paged_config* c, const int32_t* cu, int64_t total) {
  if (!cu) return GLIDE_ERR_NULL;
  if (total < 0 || cu[0] != 0 || cu[c->batch] != total) return GLIDE_ERR_INVALID;
  for (int32_t b = 0; b < c->batch; ++b)
    if (cu[b + 1] < cu[b]) return GLIDE_ERR_INVALID;
  for (int32_t b = 0; b < c->batch; ++b)
    if (int64_t(cu[b + 1] - cu[b]) * c->n_q_heads * c->head_dim * esize(c) >= (int64_t(1) << 31))
      return GLIDE_ERR_UNSUPPORTED;
  return GLIDE_OK;
}

int32_t capacity(const glide_paged_config* c) { return c->max_pages * c->page_size; }

// Tokens that one query sees at most.
int64_t most_seen(const glide_paged_config* c, int64_t max_len) {
  int64_t n = capacity(c);
  if (max_len > 0) n = std::min(n, max_len);
  return std::min<int64_t>(n, int64_t(c->window) + c->n_sinks);
}

int64_t max_pieces(int64_t tiles, int rows) {
  return std::max<int64_t>(1, std::min<int64_t>(kPagedMaxPieces, kMaxRecords / (std::max<int64_t>(tiles, 1) * rows)));
}

// Pieces of each row tile (see kPagedRound).  max_len only sizes them: the
// kernels make pieces longer where rows see more.
void set_pieces(int64_t n, int64_t keys, PagedArgs* a) {
  a->npiece = int32_t(n);
  a->piece = int32_t(((keys + n - 1) / n + 127) / 128 * 128);
}
void plan_decode(const glide_paged_config* c, int64_t max_len, PagedArgs* a) {
  const int64_t keys = std::max<int64_t>(1, most_seen(c, max_len)), units = int64_t(c->batch) * c->n_kv_heads;
  const int64_t piece = std::min<int64_t>(kPieceLong, std::max<int64_t>(kPieceMin, units * keys / kPagedRound));
  set_pieces(std::min((keys + piece - 1) / piece, max_pieces(units, kPagedRows)), keys, a);
}
// Steps of the prefill kernels, timed with one and with two workgroups per CU.
StepCost step_cost(const glide_paged_config* c, int tile_rows) {
  const double d = c->head_dim / 128.0;
  if (tile_rows == kTileRows) return {kTileKeys, 1.5, 2.1};
  if (c->dtype == GLIDE_BF16)  // pages of fewer than 16 tokens
    return tile_rows == kSharedRows ? StepCost{kPagedTile, 1.0, 1.3} : StepCost{4 * kPagedTile, 1.5 + d, 3.3};
  return tile_rows == kSharedRows ? StepCost{kPagedTile, 1.2 + 1.8 * d, 0.4 + 4.9 * d}
                                  : StepCost{4 * kPagedTile, 0.5 + 4 * d, 0.7 + 7.4 * d};
}
// The best number of pieces of a prefill of `rows` rows in `tiles` row tiles
// (nseq sequences), whose longest tile sees `keys` keys (`key_bytes` of K and V
// each), and the time that the model gives it.  coarse: of about every fifth
// number only, for less of the host's time.
double plan_pieces(const glide_paged_config* c, const StepCost& cost, int64_t tiles, int tile_rows, int64_t rows,
                   int64_t nseq, int64_t keys, double key_bytes, bool coarse, int64_t* pieces) {
  const double kv = nseq * c->n_kv_heads * double(keys) * key_bytes;
  // new tokens of a sequence, against the keys that the last of them sees
  const double T = double(rows) / (double(nseq) * c->n_q_heads), K = double(keys);
  const double avg = T <= K ? 1 - T / (2 * K) : 1 - K / (2 * T);
  auto us = [&](int64_t m) { return prefill_us(double(tiles), keys, avg, cost, m, rows, kv, c->head_dim); };
  int64_t n = 1;
  double best = us(1);
  const int64_t most = std::min((keys + cost.keys - 1) / cost.keys, max_pieces(tiles, tile_rows));
  for (int64_t m = 2; m <= most; m += coarse ? 1 + m / 4 : 1) {
    const double x = us(m);
    if (x < best) {
      n = m;
      best = x;
    }
  }
  *pieces = n;
  return best;
}
double plan_prefill(const glide_paged_config* c, int64_t tiles, int tile_rows, int64_t rows, int64_t nseq,
                    int64_t keys, int64_t* pieces) {
  return plan_pieces(c, step_cost(c, tile_rows), tiles, tile_rows, rows, nseq, keys, 2.0 * c->head_dim * esize(c),
                     false, pieces);
}

// Sections of the workspace of one call, in bytes from its start.
struct Sections {
  int64_t acc, ml, lse2, scores, bytes;
};
Sections sections(const glide_paged_config* c, int64_t rows, int64_t record_rows, bool weights, bool decode) {
  Sections s;
  s.acc = 0;
  s.ml = align256(record_rows * c->head_dim * 4);
  s.lse2 = s.ml + align256(record_rows * 2 * 4);
  s.scores = s.lse2 + (weights ? align256(rows * 4) : 0);
  const int64_t nv = (most_seen(c, 0) + 31) / 32 * 32;
  s.bytes = s.scores + (weights && decode ? align256(rows * nv * 4) : 0);
  return s;
}

// Row tiles of a prefill: of each sequence's rows.
int64_t row_tiles(const glide_paged_config* c, const int32_t* cu, int b0, int b1, int rows) {
  int64_t n = 0;
  const int G = c->n_q_heads / c->n_kv_heads;
  for (int b = b0; b < b1; ++b) n += (int64_t(cu[b + 1] - cu[b]) * G + rows - 1) / rows;
  return n;
}

// Rows per tile of a prefill.
//  attend_tiles (bf16), also where few of its 128 rows are there (it reads K
//    and V once for all of them).  It takes 16 keys of a page at 32-bit
//    offsets: pages of 16 tokens or more, no rows further apart than that.
//  Else attend_shared (64 rows, each wave 16 of them over every key) or
//    attend_rows (16 rows, each wave a quarter of the keys), whichever the
//    model gives less time.  fp32, 40 tokens onto 16000: 148 / 176 us; four
//    512-token prompts of 4 heads, d = 64, W = 64: 17.7 / 11.2 us; 600 tokens
//    61 / 72 us; bf16, pages of 4, 100 tokens onto 900: 20.6 / 26.9 us.
int tile_rows(const glide_paged_config* c, const glide_paged_cache* k, const int32_t* cu, int64_t max_len) {
  const int64_t far = int64_t(1) << 26;
  if (c->dtype == GLIDE_BF16 && c->page_size >= 16 && k->k_strides[2] <= far && k->v_strides[2] <= far)
    return kTileRows;
  const int64_t rows = int64_t(cu[c->batch]) * c->n_q_heads, keys = std::max<int64_t>(1, most_seen(c, max_len));
  int64_t nseq = 0, n;
  for (int32_t b = 0; b < c->batch; ++b) nseq += cu[b + 1] > cu[b];
  auto us = [&](int r) {
    return plan_prefill(c, std::max<int64_t>(1, row_tiles(c, cu, 0, c->batch, r) * c->n_kv_heads), r, rows, nseq, keys,
                        &n);
  };
  return us(kSharedRows) < us(kPagedRows) ? kSharedRows : kPagedRows;
}

void fill(const glide_paged_config* c, const glide_paged_cache* k, PagedArgs* a) {
  memset(a, 0, sizeof(*a));
  a->kp = static_cast<char*>(k->k);
  a->vp = static_cast<char*>(k->v);
  a->wp = k->weights;
  a->table = k->block_table;
  a->lens = k->lens;
  for (int i = 0; i < 3; ++i) {
    a->ks[i] = k->k_strides[i] * esize(c);
    a->vs[i] = k->v_strides[i] * esize(c);
  }
  a->B = c->batch;
  a->Hq = c->n_q_heads;
  a->Hkv = c->n_kv_heads;
  a->G = c->n_q_heads / c->n_kv_heads;
  a->n_pages = c->n_pages;
  a->max_pages = c->max_pages;
  a->shift = __builtin_ctz(uint32_t(c->page_size));
  a->cap = capacity(c);
  a->W = c->window;
  a->ns = c->n_sinks;
  // (a scale of 0 stays a number that no -inf becomes NaN by)
  a->scale = c->sm_scale * kLog2e;
  if (fabsf(a->scale) < 1e-30f) a->scale = 1e-30f;
}

// The sequences of one launch, from b0 on; *units: workgroups per KV head.
// per(T): those of a sequence of T new tokens.  most: rows of several sequences.
template <typename F>
int next_launch(const glide_paged_config* c, const int32_t* cu, int b0, PagedSeqs* t, F per,
                int64_t most = kMaxLaunchRows) {
  memset(t, 0, sizeof(*t));
  t->seq0 = b0;
  int b1 = b0;
  while (b1 < c->batch && b1 - b0 < kMaxSeqPerLaunch &&
         (b1 == b0 || int64_t(cu[b1 + 1] - cu[b0]) * c->n_q_heads <= most)) {
    const int i = b1 - b0;
    t->start[i] = cu[b1];
    t->len[i] = cu[b1 + 1] - cu[b1];
    t->tile0[i + 1] = t->tile0[i] + (t->len[i] ? int32_t(per(int64_t(t->len[i]))) : 0);
    ++b1;
  }
  t->nseq = b1 - b0;
  return b1;
}

glide_status hip_status(hipError_t e) { return e == hipSuccess ? GLIDE_OK : GLIDE_ERR_HIP; }

}  // namespace
}  // namespace glide
