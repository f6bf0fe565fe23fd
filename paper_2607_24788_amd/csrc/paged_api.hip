// C ABI of the paged softmax cache: argument validation (on the host, before
// the first HIP call), workspace and launch planning (paged_host.h).
#include "paged_host.h"

using namespace glide;

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
