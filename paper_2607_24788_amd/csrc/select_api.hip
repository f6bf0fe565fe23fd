// C ABI of the attention over selected pages: argument validation (on the host,
// before the first HIP call), workspace and launch planning.
#include "paged_host.h"
#include "select.h"

using namespace glide;

namespace {

// Rows of one launch at most: what their scores take in the workspace.
int64_t launch_rows(const glide_paged_config* c, int64_t rows) {
  const int64_t one = int64_t(c->n_kv_heads) * c->max_pages * 8;
  return std::min(rows, std::max<int64_t>(1, std::min(kMaxScoreBytes / one, kMaxLaunchUnits / c->n_kv_heads)));
}

struct SparseSections {
  int64_t keys, pages, held, acc, ml, bytes;
};
SparseSections sparse_sections(const glide_paged_config* c, int64_t total, int32_t n_select) {
  const int64_t R = launch_rows(c, total), units = R * c->n_kv_heads;
  const int64_t records = std::min(R * c->n_q_heads * kPagedMaxPieces, kMaxRecords);
  SparseSections s;
  s.keys = 0;
  s.pages = align256(units * c->max_pages * 8);
  s.held = s.pages + align256(units * n_select * 4);
  s.acc = s.held + align256(units * 4);
  s.ml = s.acc + align256(records * c->head_dim * 4);
  s.bytes = s.ml + align256(records * 8);
  return s;
}

bool select_fits(const glide_paged_config* c, int32_t n_select) {
  return n_select >= 1 && int64_t(n_select) * c->page_size <= kMaxPagedWindow;
}

int64_t longest_seq(const glide_paged_config* c, int64_t max_len) {
  return max_len ? std::min<int64_t>(max_len, capacity(c)) : capacity(c);
}

// The sequences of the launch that starts at row0, R rows at most, whose first
// is *b0 or a later one; returns the row behind its last.
int64_t launch_seqs(const glide_paged_config* c, const int32_t* cu, int64_t row0, int64_t R, int64_t* b0,
                    PagedSeqs* t) {
  memset(t, 0, sizeof(*t));
  while (cu[*b0 + 1] <= row0) ++*b0;  // the sequence of the first row
  t->seq0 = int32_t(*b0);
  int64_t row1 = row0;
  int i = 0;
  for (int64_t b = *b0; b < c->batch && i < kMaxSeqPerLaunch && row1 < row0 + R; ++b, ++i) {
    row1 = std::min<int64_t>(cu[b + 1], row0 + R);
    t->start[i] = cu[b];
    t->len[i] = cu[b + 1] - cu[b];
    t->tile0[i + 1] = t->tile0[i] + int32_t((row1 - std::max<int64_t>(cu[b], row0) + kScoreRows - 1) / kScoreRows);
  }
  t->nseq = i;
  return row1;
}

// How the rows row0 .. row1 - 1 of a launch are attended to (see kPickedUnits,
// kSharedUnits); u: tile0 counts picked_tiles' waves per KV head.
SparseForm sparse_form(const glide_paged_config* c, const PagedSeqs& t, int64_t row0, int64_t row1, int32_t n_select,
                       int64_t longest, PagedSeqs* u) {
  const int together = kPagedRows / (c->n_q_heads / c->n_kv_heads);  // rows of a wave
  *u = t;
  for (int x = 0; x < t.nseq; ++x) {
    const int64_t lo = std::max<int64_t>(t.start[x], row0);
    const int64_t hi = std::min<int64_t>(int64_t(t.start[x]) + t.len[x], row1);
    u->tile0[x + 1] = u->tile0[x] + int32_t((std::max<int64_t>(hi - lo, 0) + together - 1) / together);
  }
  const int64_t units = (row1 - row0) * c->n_kv_heads, waves = int64_t(u->tile0[u->nseq]) * c->n_kv_heads;
  // times that a page is selected by a wave's rows, if they choose by chance
  const double part = std::min(1.0, double(n_select) * c->page_size / double(longest));
  const double share = together * part / (1 - pow(1 - part, together));
  const bool fits = c->page_size >= 32 || (c->page_size == 16 && share * share >= together);
  if (c->dtype == GLIDE_BF16 && fits && waves >= kSharedUnits && 5 * units >= 8 * waves) return SparseForm::tiles;
  return units >= kPickedUnits ? SparseForm::waves : SparseForm::workgroups;
}

}  // namespace

extern "C" {

size_t glide_paged_sparse_workspace_bytes(const glide_paged_config* cfg, int64_t max_total_tokens, int32_t n_select) {
  if (check_cfg(cfg) != GLIDE_OK || !select_fits(cfg, n_select)) return 0;
  if (max_total_tokens < 0 || max_total_tokens > (int64_t(1) << 31)) return 0;
  return size_t(std::max<int64_t>(256, sparse_sections(cfg, max_total_tokens, n_select).bytes));
}

glide_status glide_paged_sparse(const glide_paged_config* cfg, const glide_paged_cache* cache, const void* bounds,
                                const void* q, const int32_t* cu_seqlens_host, int64_t total_tokens, int32_t n_select,
                                int32_t n_first, int32_t n_recent, int64_t max_len, int32_t* selected, void* out,
                                float* lse, void* workspace, size_t workspace_bytes, void* stream) {
  glide_status s = check_cfg(cfg);
  if (s != GLIDE_OK) return s;
  s = check_cache(cfg, cache);
  if (s != GLIDE_OK) return s;
  const int32_t* cu = cu_seqlens_host;
  s = check_cu(cfg, cu, total_tokens);
  if (s != GLIDE_OK) return s;
  if (!select_fits(cfg, n_select) || n_first < 0 || n_recent < 1 || max_len < 0) return GLIDE_ERR_INVALID;
  if (int64_t(n_first) + n_recent > n_select) return GLIDE_ERR_INVALID;
  if (total_tokens == 0) return GLIDE_OK;
  if (!bounds || !q || !selected || !out || !workspace) return GLIDE_ERR_NULL;
  if (!aligned(bounds, 16) || !aligned(q, 16) || !aligned(out, 16) || !aligned(selected, 4) || !aligned(lse, 4) ||
      !aligned(workspace, 256))
    return GLIDE_ERR_ALIGN;
  if (workspace_bytes < glide_paged_sparse_workspace_bytes(cfg, total_tokens, n_select)) return GLIDE_ERR_SIZE;

  PagedArgs a;
  fill(cfg, cache, &a);
  a.wp = nullptr;
  SelectArgs e;
  memset(&e, 0, sizeof(e));
  e.q = static_cast<const char*>(q);
  e.bounds = static_cast<const char*>(bounds);
  e.table = a.table;
  e.lens = a.lens;
  e.Hq = a.Hq;
  e.Hkv = a.Hkv;
  e.G = a.G;
  e.n_pages = a.n_pages;
  e.max_pages = a.max_pages;
  e.shift = a.shift;
  e.cap = a.cap;
  e.n_select = n_select;
  e.n_first = n_first;
  e.n_recent = n_recent;
  e.negative = cfg->sm_scale < 0;
  const SparseSections w = sparse_sections(cfg, total_tokens, n_select);
  char* ws = static_cast<char*>(workspace);
  e.keys = reinterpret_cast<uint64_t*>(ws + w.keys);
  e.selected = selected;
  e.pages = reinterpret_cast<int32_t*>(ws + w.pages);
  e.held = reinterpret_cast<int32_t*>(ws + w.held);
  // the attention: each (row, KV head) over a table of its own, the pages that were selected, all of them
  a.per_head = 1;
  a.table = e.pages;
  a.lens = e.held;
  a.max_pages = n_select;
  a.cap = n_select << a.shift;
  a.W = kMaxPagedWindow;
  a.ns = 0;
  const int64_t longest = longest_seq(cfg, max_len);
  const int64_t keys = std::min<int64_t>(a.cap, longest), R = launch_rows(cfg, total_tokens);
  for (int64_t row0 = 0, b0 = 0; row0 < total_tokens;) {
    PagedSeqs t, u;
    const int64_t row1 = launch_seqs(cfg, cu, row0, R, &b0, &t);
    e.row0 = int32_t(row0);
    e.row1 = int32_t(row1);
    e.single = t.nseq == row1 - row0 && t.tile0[t.nseq] == t.nseq;
    const int64_t pages = (longest + cfg->page_size - 1) / cfg->page_size;
    // (one token of 2047 pages: 32 pages a workgroup 20.8 us, 64 21.7; 32 of 769: 77.7, 76.7)
    const int64_t chunk = int64_t(t.tile0[t.nseq]) * cfg->n_kv_heads * pages / kScoreWorkgroups;
    e.chunk = int32_t(std::min<int64_t>(128, std::max<int64_t>(32, (chunk + 31) / 32 * 32)));
    s = hip_status(launch_select(e, t, pages, cfg->head_dim, cfg->dtype, hipStream_t(stream)));
    if (s != GLIDE_OK) return s;
    const int64_t rows = row1 - row0, units = rows * cfg->n_kv_heads, row = int64_t(cfg->n_q_heads) * cfg->head_dim;
    a.B = int32_t(rows);
    a.q = static_cast<const char*>(q) + row0 * row * esize(cfg);
    a.out = static_cast<char*>(out) + row0 * row * esize(cfg);
    a.lse = lse ? lse + row0 * cfg->n_q_heads : nullptr;
    a.acc = reinterpret_cast<float*>(ws + w.acc);
    a.ml = reinterpret_cast<float*>(ws + w.ml);
    const SparseForm form = sparse_form(cfg, t, row0, row1, n_select, longest, &u);
    if (form == SparseForm::tiles) {
      PagedArgs o = a;
      o.table = e.table;
      o.lens = e.lens;
      o.max_pages = e.max_pages;
      o.cap = e.cap;
      s = hip_status(launch_picked_tiles(o, u, e, kPagedRows / a.G, cfg->head_dim, hipStream_t(stream)));
    } else if (form == SparseForm::waves) {
      s = hip_status(launch_picked(a, int32_t(units), cfg->head_dim, cfg->dtype, hipStream_t(stream)));
    } else {
      // Pieces for a round of workgroups, none where every CU has one without: 8
      // units of 4096 keys, 128 / 256 keys a piece 20.8 / 22.4 us; 192 of 2112, two
      // pieces 49.5, three 56, one 54; 256 of 2048, one 76.5, two 77.7.
      const int64_t split = units >= kPagedRound / 2 ? 1 : kPagedRound / units;
      set_pieces(std::min(split, std::min((keys + kPieceMin - 1) / kPieceMin, max_pieces(units, kPagedRows))), keys,
                 &a);
      s = hip_status(launch_paged_decode(a, keys, cfg->head_dim, cfg->dtype, hipStream_t(stream)));
    }
    if (s != GLIDE_OK) return s;
    row0 = row1;
  }
  return GLIDE_OK;
}

int32_t glide_internal_sparse_form(const glide_paged_config* cfg, const int32_t* cu, int32_t n_select,
                                   int64_t max_len) {
  PagedSeqs t, u;
  int64_t b0 = 0;
  const int64_t row1 = launch_seqs(cfg, cu, 0, launch_rows(cfg, cu[cfg->batch]), &b0, &t);
  return int32_t(sparse_form(cfg, t, 0, row1, n_select, longest_seq(cfg, max_len), &u));
}

}  // extern "C"
