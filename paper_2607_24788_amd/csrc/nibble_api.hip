// C ABI of the attention over a 4-bit paged cache: argument validation (on the
// host, before the first HIP call), workspace and launch planning.
#include "nibble.h"
#include "paged_host.h"

using namespace glide;

namespace {

void fill4(const glide_paged_config* c, const glide_nibble_cache* k, PagedArgs* a, Pools4* p) {
  glide_paged_cache none;
  memset(&none, 0, sizeof(none));
  none.block_table = k->block_table;
  none.lens = k->lens;
  fill(c, &none, a);
  *p = {k->k_codes, k->k_scales, k->v_codes, k->v_scales};
}

double key_bytes4(const glide_paged_config* c) { return 2.0 * (c->head_dim / 2 + c->head_dim / kGroup4); }

// Steps of the prefill kernels, timed with half a round of workgroups and with
// whole ones; a CU holds two workgroups of nibble_rows and of 128 rows in bf16,
// one of the others.
StepCost step_cost4(const glide_paged_config* c, int tile_rows) {
  const bool wide = c->head_dim == 128;
  if (c->dtype == GLIDE_BF16) {
    if (tile_rows == kPagedRows) return {256, wide ? 2.2 : 1.6, wide ? 2.85 : 2.2, kPagedRound, 3.5};
    if (tile_rows == kRows4) return {kTileKeys, wide ? 1.35 : 0.8, wide ? 2.15 : 1.15, kPagedRound, 3.5};
    return {kTileKeys, wide ? 1.75 : 1.3, wide ? 1.98 : 1.3, kPagedRound / 2, 4.5};
  }
  if (tile_rows == kPagedRows) return {256, wide ? 2.6 : 2.0, wide ? 3.7 : 2.8, kPagedRound, 4};
  if (tile_rows == kRows4) return {kTileKeys, wide ? 2.8 : 1.6, wide ? 2.95 : 1.7, kPagedRound / 2, 6};
  return {kTileKeys, wide ? 3.6 : 2.4, wide ? 4.3 : 2.5, kPagedRound / 2, 6};
}

// Rows per workgroup of a prefill: what the model gives least time, of a
// launch's rows.  More rows share the conversion of a tile; fewer leave a CU's
// waves to more of the keys.  128 / 256 rows, 32 / 8 heads of 128, bf16: 32768
// tokens 8.35 / 8.13 ms, 1024 fresh ones 28.7 / 35.9 us; fp32, 4096 tokens 401
// / 315 us; 16 / 128 rows: 5 tokens onto 8000 13.8 / 14.2 us, one fp32 layer of
// 512 tokens and W = 64 7.4 / 14.6 us.
int tile_rows4(const glide_paged_config* c, const int32_t* cu, int b0, int b1, int64_t max_len, int64_t* pieces,
               int64_t* keys) {
  const int G = c->n_q_heads / c->n_kv_heads;
  const int64_t rows = int64_t(cu[b1] - cu[b0]) * c->n_q_heads, most = most_seen(c, max_len);
  const int64_t all = max_len > 0 ? std::min<int64_t>(max_len, capacity(c)) : capacity(c);
  int64_t nseq = 0, longest = 0;
  for (int b = b0; b < b1; ++b) {
    nseq += cu[b + 1] > cu[b];
    longest = std::max<int64_t>(longest, cu[b + 1] - cu[b]);
  }
  int best = kPagedRows;
  double least = 0;
  for (int r : {kPagedRows, kRows4, kRows4Big}) {
    // the longest tile sees what its first and its last row do
    const int64_t k = std::max<int64_t>(1, std::min(all, most + std::min<int64_t>((r + G - 1) / G, longest) - 1));
    const int64_t tiles = std::max<int64_t>(1, row_tiles(c, cu, b0, b1, r) * c->n_kv_heads);
    int64_t n;
    const double us = plan_pieces(c, step_cost4(c, r), tiles, r, rows, std::max<int64_t>(1, nseq), k, key_bytes4(c),
                                  true, &n);
    if (r == kPagedRows || us < least) {
      best = r;
      least = us;
      *pieces = n;
      *keys = k;
    }
  }
  return best;
}

// Pieces of the rows of a decode; returns the keys of a wave's tile.  Times by
// keys of a piece, bf16, 32 / 8 heads of 128 where not said:
//  Rows of 1024 keys or fewer are not split: 500 keys 7.8 us whole, 9.0 in two.
//  Large calls (bf16, d = 128): tiles of 32 keys, four workgroups to a CU and
//    pieces for one round of them, 4096 keys at most (a workgroup's start and
//    end weigh more than what shorter pieces even out): 8 sequences of 32768,
//    1024 / 2048 / 4096 keys 55 / 50 / 54 us; 32 of 16384 .. 32768, 512 / 4096
//    161 / 151 us (tiles of 64 keys, two to a CU: 192 / 168).
//  d = 64: tiles of 32 keys where rows of up to 512 keys are more than three
//    workgroups to a CU, which is what tiles of 64 have at once: 784 rows of 300
//    keys 8.2 us (64: 10.6), 1024 of 300 8.4 (10.9), 2048 of 300 16.0 (19.6), of 1
//    .. 500 17.0 (18.8), 1520 of 500 16.9 (16.2).  Beyond: 768 of 700 11.8 (10.9),
//    1056 of 700 18.8 (17.6), 1024 of 100 .. 4000 45.5 (44); in pieces, 16
//    sequences of 20000 41 (41), 96 of 500 .. 40000 with W = 8192 105 (96).
//  Where that would leave pieces under kSmall4 keys, and for the others (fp32 among
//    them): tiles of 64 keys, two workgroups to a CU.  One sequence of 32768:
//    512 keys 14.1 us (tiles of 32: 256 keys 16.8); of 8192: 256 keys 9.6 us,
//    512 10.6 (tiles of 32: 10.0).
int plan_decode4(const glide_paged_config* c, int64_t max_len, PagedArgs* a) {
  constexpr int64_t kWhole4 = 1024, kSmall4 = 384, kLeast4 = 256, kMost4 = 4096;
  const int64_t keys = std::max<int64_t>(1, most_seen(c, max_len)), units = int64_t(c->batch) * c->n_kv_heads;
  const int64_t all = units * keys;
  const bool many = c->head_dim == 128 ? all >= kSmall4 * 2 * kPagedRound : units > kPagedRound * 3 / 2 && keys <= 512;
  const bool large = c->dtype == GLIDE_BF16 && many;
  int64_t piece = std::min(kMost4, std::max(kLeast4, all / (large ? 2 * kPagedRound : kPagedRound)));
  if (keys <= kWhole4) piece = keys;
  set_pieces(std::min((keys + piece - 1) / piece, max_pieces(units, kPagedRows)), keys, a);
  return large ? 32 : 64;
}

}  // namespace

extern "C" {

size_t glide_nibble_workspace_bytes(const glide_paged_config* cfg, int64_t max_total_tokens) {
  return glide_paged_workspace_bytes(cfg, max_total_tokens, 0);
}

glide_status glide_nibble_prefill(const glide_paged_config* cfg, const glide_nibble_cache* cache, const void* q,
                                  const int32_t* cu_seqlens_host, int64_t total_tokens, int64_t max_len, void* out,
                                  float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache4(cfg, cache);
  if (s != GLIDE_OK) return s;
  const int32_t* cu = cu_seqlens_host;
  s = check_cu(cfg, cu, total_tokens);
  if (s != GLIDE_OK) return s;
  if (max_len < 0) return GLIDE_ERR_INVALID;
  if (total_tokens == 0) return GLIDE_OK;
  if (!q || !out || !workspace) return GLIDE_ERR_NULL;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(workspace, 256)) return GLIDE_ERR_ALIGN;
  if (workspace_bytes < glide_nibble_workspace_bytes(cfg, total_tokens)) return GLIDE_ERR_SIZE;

  PagedArgs a;
  Pools4 p;
  fill4(cfg, cache, &a, &p);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  for (int b0 = 0; b0 < cfg->batch;) {
    PagedSeqs t;
    int b1 = next_launch(cfg, cu, b0, &t, [](int64_t) { return 0; });
    int64_t n, keys;
    const int per_tile = tile_rows4(cfg, cu, b0, b1, max_len, &n, &keys);
    b1 = next_launch(cfg, cu, b0, &t, [&](int64_t T) { return (T * a.G + per_tile - 1) / per_tile; });
    const int64_t row0 = int64_t(cu[b0]) * cfg->n_q_heads, rows = int64_t(cu[b1]) * cfg->n_q_heads - row0;
    set_pieces(n, keys, &a);
    const Sections w = sections(cfg, total_tokens * cfg->n_q_heads, a.npiece > 1 ? rows * a.npiece : 0, false, false);
    if (size_t(w.bytes) > workspace_bytes) return GLIDE_ERR_SIZE;
    char* ws = static_cast<char*>(workspace);
    a.acc = reinterpret_cast<float*>(ws + w.acc) - row0 * a.npiece * cfg->head_dim;
    a.ml = reinterpret_cast<float*>(ws + w.ml) - row0 * a.npiece * 2;
    s = hip_status(launch_nibble_prefill(a, p, t, cfg->head_dim, cfg->dtype, per_tile, hipStream_t(stream)));
    if (s != GLIDE_OK) return s;
    b0 = b1;
  }
  return GLIDE_OK;
}

glide_status glide_nibble_decode(const glide_paged_config* cfg, const glide_nibble_cache* cache, const void* q,
                                 int64_t max_len, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache4(cfg, cache);
  if (s != GLIDE_OK) return s;
  if (!q || !out || !workspace) return GLIDE_ERR_NULL;
  if (max_len < 0) return GLIDE_ERR_INVALID;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(workspace, 256)) return GLIDE_ERR_ALIGN;
  if (workspace_bytes < glide_nibble_workspace_bytes(cfg, 0)) return GLIDE_ERR_SIZE;

  PagedArgs a;
  Pools4 p;
  fill4(cfg, cache, &a, &p);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  const int64_t rows = int64_t(cfg->batch) * cfg->n_q_heads;
  const int tile = plan_decode4(cfg, max_len, &a);
  const Sections w = sections(cfg, rows, a.npiece > 1 ? rows * a.npiece : 0, false, true);
  if (size_t(w.bytes) > workspace_bytes) return GLIDE_ERR_SIZE;
  char* ws = static_cast<char*>(workspace);
  a.acc = reinterpret_cast<float*>(ws + w.acc);
  a.ml = reinterpret_cast<float*>(ws + w.ml);
  return hip_status(launch_nibble_decode(a, p, cfg->head_dim, cfg->dtype, tile, hipStream_t(stream)));
}

int32_t glide_internal_nibble_plan(const glide_paged_config* cfg, const int32_t* cu, int64_t max_len,
                                   int32_t* pieces) {
  if (!cu) {
    PagedArgs a;
    const int tile = plan_decode4(cfg, max_len, &a);
    *pieces = a.npiece;
    return tile;
  }
  PagedSeqs t;
  const int b1 = next_launch(cfg, cu, 0, &t, [](int64_t) { return 0; });
  int64_t n, keys;
  const int rows = tile_rows4(cfg, cu, 0, b1, max_len, &n, &keys);
  *pieces = int32_t(n);
  return rows;
}

}  // extern "C"
