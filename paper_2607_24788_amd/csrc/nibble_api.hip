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
  const int per_tile = kPagedRows;
  for (int b0 = 0; b0 < cfg->batch;) {
    PagedSeqs t;
    const int b1 = next_launch(cfg, cu, b0, &t, [&](int64_t T) { return (T * a.G + per_tile - 1) / per_tile; });
    const int64_t row0 = int64_t(cu[b0]) * cfg->n_q_heads, rows = int64_t(cu[b1]) * cfg->n_q_heads - row0;
    const int64_t keys = std::max<int64_t>(1, most_seen(cfg, max_len));
    int64_t n;
    plan_prefill(cfg, std::max<int64_t>(1, int64_t(t.tile0[t.nseq]) * cfg->n_kv_heads), per_tile, rows, t.nseq, keys,
                 &n);
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
  plan_decode(cfg, max_len, &a);
  const Sections w = sections(cfg, rows, a.npiece > 1 ? rows * a.npiece : 0, false, true);
  if (size_t(w.bytes) > workspace_bytes) return GLIDE_ERR_SIZE;
  char* ws = static_cast<char*>(workspace);
  a.acc = reinterpret_cast<float*>(ws + w.acc);
  a.ml = reinterpret_cast<float*>(ws + w.ml);
  return hip_status(launch_nibble_decode(a, p, cfg->head_dim, cfg->dtype, hipStream_t(stream)));
}

}  // extern "C"
