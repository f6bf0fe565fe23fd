// C ABI of the paged softmax cache: argument validation (on the host, before
// the first HIP call), workspace and launch planning.
#include <math.h>
#include <string.h>

#include <algorithm>

#include "paged.h"

using namespace glide;

namespace {

constexpr int32_t kMaxPagedWindow = 1 << 30;
constexpr int32_t kMaxSinks = 1 << 20;
constexpr int64_t kMaxUnits = int64_t(1) << 20;       // B * Hkv, a grid dimension
constexpr int64_t kMaxLaunchRows = int64_t(1) << 27;  // rows of one prefill launch

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
// (nseq sequences), and the time that the model gives it.
double plan_prefill(const glide_paged_config* c, int64_t tiles, int tile_rows, int64_t rows, int64_t nseq,
                    int64_t keys, int64_t* pieces) {
  const StepCost cost = step_cost(c, tile_rows);
  const double kv = 2.0 * nseq * c->n_kv_heads * double(keys) * c->head_dim * esize(c);
  // new tokens of a sequence, against the keys that the last of them sees
  const double T = double(rows) / (double(nseq) * c->n_q_heads), K = double(keys);
  const double avg = T <= K ? 1 - T / (2 * K) : 1 - K / (2 * T);
  auto us = [&](int64_t m) { return prefill_us(double(tiles), keys, avg, cost, m, rows, kv, c->head_dim); };
  int64_t n = 1;
  double best = us(1);
  const int64_t most = std::min((keys + cost.keys - 1) / cost.keys, max_pieces(tiles, tile_rows));
  for (int64_t m = 2; m <= most; ++m) {
    const double x = us(m);
    if (x < best) {
      n = m;
      best = x;
    }
  }
  *pieces = n;
  return best;
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

glide_status hip_status(hipError_t e) { return e == hipSuccess ? GLIDE_OK : GLIDE_ERR_HIP; }

}  // namespace

extern "C" {

size_t glide_paged_workspace_bytes(const glide_paged_config* cfg, int64_t max_total_tokens, int32_t weights) {
  if (check_cfg(cfg) != GLIDE_OK || max_total_tokens < 0) return 0;
  if (max_total_tokens > (int64_t(1) << 31)) return 0;
  const int64_t rows = int64_t(cfg->batch) * cfg->n_q_heads, units = int64_t(cfg->batch) * cfg->n_kv_heads;
  const int64_t np = max_pieces(units, kPagedRows);
  int64_t n = sections(cfg, rows, np > 1 || weights ? rows * np : 0, weights, true).bytes;
  const int64_t prows = max_total_tokens * cfg->n_q_heads;
  n = std::max(n, sections(cfg, prows, std::min(prows * kPagedMaxPieces, kMaxRecords), weights, false).bytes);
  return size_t(std::max<int64_t>(256, n));
}

glide_status glide_paged_prefill(const glide_paged_config* cfg, const glide_paged_cache* cache, const void* q,
                                 const void* k, const void* v, const int32_t* cu_seqlens_host, int64_t total_tokens,
                                 int32_t n_observe, int64_t max_len, void* out, float* lse, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache(cfg, cache);
  if (s != GLIDE_OK) return s;
  if (!cu_seqlens_host) return GLIDE_ERR_NULL;
  const int32_t* cu = cu_seqlens_host;
  if (total_tokens < 0 || n_observe < 0 || max_len < 0) return GLIDE_ERR_INVALID;
  if (cu[0] != 0 || cu[cfg->batch] != total_tokens) return GLIDE_ERR_INVALID;
  for (int32_t b = 0; b < cfg->batch; ++b)
    if (cu[b + 1] < cu[b]) return GLIDE_ERR_INVALID;
  if (n_observe > 0 && !cache->weights) return GLIDE_ERR_NULL;
  if (!k != !v) return GLIDE_ERR_NULL;
  for (int32_t b = 0; b < cfg->batch; ++b)
    if (int64_t(cu[b + 1] - cu[b]) * cfg->n_q_heads * cfg->head_dim * esize(cfg) >= (int64_t(1) << 31))
      return GLIDE_ERR_UNSUPPORTED;
  if (total_tokens == 0) return GLIDE_OK;
  if (!q || !out || !workspace) return GLIDE_ERR_NULL;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lse, 4) ||
      !aligned(workspace, 256))
    return GLIDE_ERR_ALIGN;
  if (workspace_bytes < glide_paged_workspace_bytes(cfg, total_tokens, n_observe > 0)) return GLIDE_ERR_SIZE;

  PagedArgs a;
  fill(cfg, cache, &a);
  a.q = static_cast<const char*>(q);
  a.kn = static_cast<const char*>(k);
  a.vn = static_cast<const char*>(v);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  hipStream_t st = hipStream_t(stream);
  const int per_tile = tile_rows(cfg, cache, cu, max_len);
  for (int b0 = 0; b0 < cfg->batch;) {
    PagedSeqs t;
    memset(&t, 0, sizeof(t));
    t.seq0 = b0;
    int b1 = b0;
    while (b1 < cfg->batch && b1 - b0 < kMaxSeqPerLaunch &&
           (b1 == b0 || int64_t(cu[b1 + 1] - cu[b0]) * cfg->n_q_heads <= kMaxLaunchRows)) {
      const int i = b1 - b0;
      t.start[i] = cu[b1];
      t.len[i] = cu[b1 + 1] - cu[b1];
      t.tile0[i + 1] = t.tile0[i] + int32_t(row_tiles(cfg, cu, b1, b1 + 1, per_tile));
      ++b1;
    }
    t.nseq = b1 - b0;
    // records by the call's row number: a launch's own rows only
    const int64_t row0 = int64_t(cu[b0]) * cfg->n_q_heads, rows = int64_t(cu[b1]) * cfg->n_q_heads - row0;
    const int64_t keys = std::max<int64_t>(1, most_seen(cfg, max_len));
    int64_t n;
    plan_prefill(cfg, std::max<int64_t>(1, int64_t(t.tile0[t.nseq]) * cfg->n_kv_heads), per_tile, rows, t.nseq, keys,
                 &n);
    set_pieces(n, keys, &a);
    const Sections w = sections(cfg, total_tokens * cfg->n_q_heads, a.npiece > 1 ? rows * a.npiece : 0,
                                n_observe > 0, false);
    char* ws = static_cast<char*>(workspace);
    a.acc = reinterpret_cast<float*>(ws + w.acc) - row0 * a.npiece * cfg->head_dim;
    a.ml = reinterpret_cast<float*>(ws + w.ml) - row0 * a.npiece * 2;
    a.lse2 = n_observe > 0 ? reinterpret_cast<float*>(ws + w.lse2) : nullptr;
    if (size_t(w.bytes) > workspace_bytes) return GLIDE_ERR_SIZE;
    s = hip_status(launch_paged_prefill(a, t, cfg->head_dim, cfg->dtype, per_tile, st));
    if (s != GLIDE_OK) return s;
    if (n_observe > 0) {
      int32_t longest = 0;
      for (int i = 0; i < t.nseq; ++i) longest = std::max(longest, t.len[i]);
      const int64_t seen = std::min<int64_t>(capacity(cfg), int64_t(cfg->window) + cfg->n_sinks +
                                                                std::min(longest, n_observe));
      s = hip_status(launch_paged_weights(a, t, n_observe, seen, cfg->head_dim, cfg->dtype, st));
      if (s != GLIDE_OK) return s;
    }
    b0 = b1;
  }
  return GLIDE_OK;
}

glide_status glide_paged_decode(const glide_paged_config* cfg, const glide_paged_cache* cache, const void* q,
                                const void* k, const void* v, int64_t max_len, void* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache(cfg, cache);
  if (s != GLIDE_OK) return s;
  if (!q || !out || !workspace || !k != !v) return GLIDE_ERR_NULL;
  if (max_len < 0) return GLIDE_ERR_INVALID;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(lse, 4) ||
      !aligned(workspace, 256))
    return GLIDE_ERR_ALIGN;
  const bool weights = cache->weights != nullptr;
  if (workspace_bytes < glide_paged_workspace_bytes(cfg, 0, weights)) return GLIDE_ERR_SIZE;

  PagedArgs a;
  fill(cfg, cache, &a);
  a.q = static_cast<const char*>(q);
  a.kn = static_cast<const char*>(k);
  a.vn = static_cast<const char*>(v);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  const int64_t rows = int64_t(cfg->batch) * cfg->n_q_heads;
  plan_decode(cfg, max_len, &a);
  const Sections w = sections(cfg, rows, a.npiece > 1 || weights ? rows * a.npiece : 0, weights, true);
  if (size_t(w.bytes) > workspace_bytes) return GLIDE_ERR_SIZE;
  char* ws = static_cast<char*>(workspace);
  a.acc = reinterpret_cast<float*>(ws + w.acc);
  a.ml = reinterpret_cast<float*>(ws + w.ml);
  if (weights) {
    a.scores = reinterpret_cast<float*>(ws + w.scores);
    a.nv = (most_seen(cfg, 0) + 31) / 32 * 32;
  }
  return hip_status(launch_paged_decode(a, std::max<int64_t>(1, most_seen(cfg, max_len)), cfg->head_dim, cfg->dtype,
                                        hipStream_t(stream)));
}

glide_status glide_paged_evict(const glide_paged_config* cfg, const glide_paged_cache* cache, int32_t budget,
                               int32_t n_recent, const int32_t* dst_table, int32_t* kept, int32_t* new_lens,
                               void* workspace, size_t workspace_bytes, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache(cfg, cache);
  if (s != GLIDE_OK) return s;
  if (!cache->weights || !kept || !new_lens || !workspace) return GLIDE_ERR_NULL;
  if (!aligned(dst_table, 4) || !aligned(kept, 4) || !aligned(new_lens, 4) || !aligned(workspace, 256))
    return GLIDE_ERR_ALIGN;
  if (budget < 1 || budget > kMaxPagedWindow || n_recent < 0 || int64_t(budget) < int64_t(cfg->n_sinks) + n_recent) return GLIDE_ERR_INVALID;
  if (workspace_bytes < 256) return GLIDE_ERR_SIZE;
  PagedArgs p;
  fill(cfg, cache, &p);
  EvictArgs a;
  memset(&a, 0, sizeof(a));
  a.kp = p.kp;
  a.vp = p.vp;
  a.wp = p.wp;
  a.table = p.table;
  a.lens = p.lens;
  a.dst = dst_table ? dst_table : cache->block_table;
  a.in_place = a.dst == cache->block_table;
  memcpy(a.ks, p.ks, sizeof(a.ks));
  memcpy(a.vs, p.vs, sizeof(a.vs));
  a.B = cfg->batch;
  a.Hkv = cfg->n_kv_heads;
  a.d = cfg->head_dim;
  a.esize = esize(cfg);
  a.n_pages = p.n_pages;
  a.max_pages = p.max_pages;
  a.shift = p.shift;
  a.cap = p.cap;
  a.ns = cfg->n_sinks;
  a.budget = budget;
  a.recent = n_recent;
  a.kept = kept;
  a.new_lens = new_lens;
  return hip_status(launch_paged_evict(a, hipStream_t(stream)));
}

}  // extern "C"
