// C ABI of the calls that fill a paged cache: argument validation (on the host,
// before the first HIP call) and launch planning.
#include "append.h"
#include "paged_host.h"

using namespace glide;

namespace {

glide_status check_rotation(const glide_paged_config* c, const glide_rotation* r, bool four) {
  if (!r) return GLIDE_OK;
  if (r->rot_dim < 0 || r->rot_dim > c->head_dim || r->rot_dim % 16) return GLIDE_ERR_INVALID;
  if (r->interleaved != 0 && r->interleaved != 1) return GLIDE_ERR_INVALID;
  if (four && !r->interleaved && r->rot_dim % 64) return GLIDE_ERR_UNSUPPORTED;
  if (r->rot_dim && !r->freqs) return GLIDE_ERR_NULL;
  if (!aligned(r->freqs, 16) || !aligned(r->positions, 4)) return GLIDE_ERR_ALIGN;
  return GLIDE_OK;
}

void fill_append(const glide_paged_config* c, const int32_t* table, const int32_t* lens, AppendArgs* a) {
  memset(a, 0, sizeof(*a));
  a->table = table;
  a->lens = lens;
  a->B = c->batch;
  a->Hq = c->n_q_heads;
  a->Hkv = c->n_kv_heads;
  a->G = c->n_q_heads / c->n_kv_heads;
  a->n_pages = c->n_pages;
  a->max_pages = c->max_pages;
  a->shift = __builtin_ctz(uint32_t(c->page_size));
  a->cap = capacity(c);
}
void fill_pools(const glide_paged_config* c, const glide_paged_cache* k, AppendArgs* a) {
  a->kp = static_cast<char*>(k->k);
  a->vp = static_cast<char*>(k->v);
  a->wp = k->weights;
  for (int i = 0; i < 3; ++i) {
    a->ks[i] = k->k_strides[i] * esize(c);
    a->vs[i] = k->v_strides[i] * esize(c);
  }
}

// log2 of the tokens of a workgroup where a page need not be one workgroup's:
// fewer where there would be few workgroups (512 tokens, 32 / 8 heads of 128:
// units of 64 / 16 tokens 9.4 / 5.6 us).
int32_t append_unit(const glide_paged_config* c, int64_t total) {
  int32_t unit = __builtin_ctz(uint32_t(kAppendTokens));
  while (unit > 2 && (total * c->n_kv_heads >> unit) < (unit > 4 ? 4 * kPagedRound : kPagedRound / 2)) --unit;
  return unit;
}

// An append, its cache checked and filled in.
glide_status append(const glide_paged_config* c, const glide_rotation* rot, const void* q, const void* k,
                    const void* v, const int32_t* cu, int64_t total, void* q_out, AppendArgs a, bool four,
                    void* stream) {
  glide_status s = check_rotation(c, rot, four);
  if (s != GLIDE_OK) return s;
  s = check_cu(c, cu, total);
  if (s != GLIDE_OK) return s;
  if (total == 0) return GLIDE_OK;
  if (!k || !v || !q != !q_out) return GLIDE_ERR_NULL;
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16)) return GLIDE_ERR_ALIGN;
  a.q = static_cast<const char*>(q);
  a.k = static_cast<const char*>(k);
  a.v = static_cast<const char*>(v);
  a.qo = static_cast<char*>(q_out);
  if (rot) {
    a.rot = rot->rot_dim;
    a.freqs = rot->freqs;
    a.pos = rot->positions;
  }
  // Bounds by the append itself, a page to a workgroup, where that makes enough
  // workgroups or each has few rows (one token, 192 rows); else from the keys in
  // the cache, by a launch of its own.  512 tokens, 32 / 8 heads, pages of 256:
  // 34 us / 11.9 apart, of 64: 13.2 / 10.7; 4 heads, pages of 32: 7.9 / 9.7.
  int64_t longest = 0;
  for (int32_t b = 0; b < c->batch; ++b) longest = std::max<int64_t>(longest, cu[b + 1] - cu[b]);
  AppendArgs after = a;
  const bool apart = a.bounds && longest > 1 && (total * c->n_kv_heads >> a.shift) < kPagedRound &&
                     std::min<int64_t>(longest, c->page_size) * (a.G + 2) > 192;
  if (apart) a.bounds = nullptr;
  a.unit = a.bounds ? a.shift : append_unit(c, total);
  // positions p0 .. p0 + T - 1 lie in so many units, wherever p0 is
  auto units = [](int64_t T, int32_t unit) { return ((T + (int64_t(1) << unit) - 2) >> unit) + 1; };
  for (int b0 = 0; b0 < c->batch;) {
    PagedSeqs t;
    const int b1 = next_launch(c, cu, b0, &t, [&](int64_t T) { return units(T, a.unit); }, kMaxLaunchUnits);
    s = hip_status(launch_append(a, t, c->head_dim, c->dtype, four, rot && rot->interleaved, hipStream_t(stream)));
    if (s == GLIDE_OK && apart) {
      next_launch(c, cu, b0, &t, [&](int64_t T) { return units(T, a.shift); }, kMaxLaunchUnits);
      s = hip_status(launch_new_bounds(after, t, c->head_dim, c->dtype, hipStream_t(stream)));
    }
    if (s != GLIDE_OK) return s;
    b0 = b1;
  }
  return GLIDE_OK;
}

}  // namespace

extern "C" {

glide_status glide_paged_append(const glide_paged_config* cfg, const glide_paged_cache* cache,
                                const glide_rotation* rotation, const void* q, const void* k, const void* v,
                                const int32_t* cu_seqlens_host, int64_t total_tokens, void* q_out, void* bounds,
                                void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache(cfg, cache);
  if (s != GLIDE_OK) return s;
  if (!aligned(bounds, 16)) return GLIDE_ERR_ALIGN;
  AppendArgs a;
  fill_append(cfg, cache->block_table, cache->lens, &a);
  fill_pools(cfg, cache, &a);
  a.bounds = static_cast<char*>(bounds);
  return append(cfg, rotation, q, k, v, cu_seqlens_host, total_tokens, q_out, a, false, stream);
}

glide_status glide_paged_bounds(const glide_paged_config* cfg, const glide_paged_cache* cache, int64_t max_len,
                                void* bounds, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache(cfg, cache);
  if (s != GLIDE_OK) return s;
  if (!bounds) return GLIDE_ERR_NULL;
  if (max_len < 0) return GLIDE_ERR_INVALID;
  if (!aligned(bounds, 16)) return GLIDE_ERR_ALIGN;
  AppendArgs a;
  fill_append(cfg, cache->block_table, cache->lens, &a);
  fill_pools(cfg, cache, &a);
  a.bounds = static_cast<char*>(bounds);
  const int64_t keys = max_len ? std::min<int64_t>(max_len, capacity(cfg)) : capacity(cfg);
  return hip_status(launch_page_bounds(a, keys, cfg->head_dim, cfg->dtype, hipStream_t(stream)));
}

glide_status glide_nibble_append(const glide_paged_config* cfg, const glide_nibble_cache* cache,
                                 const glide_rotation* rotation, const void* q, const void* k, const void* v,
                                 const int32_t* cu_seqlens_host, int64_t total_tokens, void* q_out, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache4(cfg, cache);
  if (s != GLIDE_OK) return s;
  AppendArgs a;
  fill_append(cfg, cache->block_table, cache->lens, &a);
  a.p4 = {cache->k_codes, cache->k_scales, cache->v_codes, cache->v_scales};
  return append(cfg, rotation, q, k, v, cu_seqlens_host, total_tokens, q_out, a, true, stream);
}

glide_status glide_nibble_read(const glide_paged_config* cfg, const glide_nibble_cache* cache,
                               const int32_t* cu_seqlens_host, int64_t total_tokens, void* k_out, void* v_out,
                               void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache4(cfg, cache);
  if (s != GLIDE_OK) return s;
  s = check_cu(cfg, cu_seqlens_host, total_tokens);
  if (s != GLIDE_OK) return s;
  if (total_tokens == 0) return GLIDE_OK;
  if (!k_out || !v_out) return GLIDE_ERR_NULL;
  if (!aligned(k_out, 16) || !aligned(v_out, 16)) return GLIDE_ERR_ALIGN;
  AppendArgs a;
  fill_append(cfg, cache->block_table, cache->lens, &a);
  a.p4 = {cache->k_codes, cache->k_scales, cache->v_codes, cache->v_scales};
  a.unit = append_unit(cfg, total_tokens);
  for (int b0 = 0; b0 < cfg->batch;) {
    PagedSeqs t;
    b0 = next_launch(cfg, cu_seqlens_host, b0, &t, [&](int64_t T) { return (T + (int64_t(1) << a.unit) - 1) >> a.unit; });
    s = hip_status(launch_read4(a, t, static_cast<char*>(k_out), static_cast<char*>(v_out), cfg->head_dim, cfg->dtype,
                                hipStream_t(stream)));
    if (s != GLIDE_OK) return s;
  }
  return GLIDE_OK;
}

}  // extern "C"
