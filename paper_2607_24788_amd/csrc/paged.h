// Launch descriptors of the paged softmax cache (kernels in paged.hip and
// evict.hip, host side in paged_api.hip).
#pragma once

#include "glide_internal.h"

namespace glide {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// A running maximum before any score: finite, so that (score - maximum) is
// never inf - inf; every real score lies far above it.
constexpr float kNoMax = -1e30f;

// Rows of one workgroup of attend_rows: one MFMA tile of (token, head) pairs.
constexpr int kPagedRows = 16;
// Rows of one workgroup of attend_tiles (four waves of 32), keys of its tiles.
constexpr int kTileRows = 128;
constexpr int kTileKeys = 64;
// Rows of one workgroup of attend_shared (four waves of 16).
constexpr int kSharedRows = 64;
// Keys of one tile of a wave of attend_rows, and of attend_shared.
constexpr int kPagedTile = 32;
// Pieces: long rows are split over workgroups and joined.  A round of
// workgroups is two per CU.
//  decode: pieces as short as one round allows (at least kPieceMin keys, a tile
//    per wave); where one round would make them longer than kPieceLong there
//    are several rounds, which even out ragged lengths.
//  prefill: by a model of the call (prefill_us).
// The records of a call are at most kMaxRecords rows.
constexpr int kPagedRound = 512;
constexpr int kPieceMin = 128;
constexpr int kPieceLong = 1024;
constexpr int kPagedMaxPieces = 256;
constexpr int64_t kMaxRecords = 131072;

// Microseconds of a prefill in n pieces per row tile, for choosing n.  Steps of
// a workgroup, one after another, take us1 each where it has a CU to itself and
// us2 where two share it; row tiles see `avg` of the longest one's keys on
// average (half in a fresh prompt), so short tiles have fewer pieces; the
// workgroups run in rounds, or (the longest first) one into another with half a
// piece of them uneven at the end.  No less than K and V at 5 TB/s, drawn by as
// many workgroups as the rounds hold on average; and the join, a launch and the
// records written and read (8 bytes per row and element at 4 TB/s).
// Measured: 16 tokens onto 500 (8 KV heads), one piece 19.5 us, four 12.1;
// 1024 fresh tokens, two pieces 55 us, one 30; 3..9 tokens onto 32K (4
// sequences), 23 pieces (1.4 rounds) 115 us, 16 (one) 100.
struct StepCost {
  int keys;
  double us1, us2;
  int round = kPagedRound;  // workgroups of a round
  double wg = 0;            // and the start and end of a workgroup, in each
};
inline double prefill_us(double tiles, int64_t keys, double avg, const StepCost& c, int64_t n, int64_t rows,
                         double kv_bytes, int d) {
  const int64_t steps = (keys + c.keys - 1) / c.keys;
  const double per = double((steps + n - 1) / n), wgs = tiles * (double(n) * avg + (1 - avg));
  const double rounds = double(int64_t((wgs + c.round - 1) / c.round));
  double t = rounds * per;
  const double even = tiles * double(steps) * avg / c.round + per / 2;
  t = t < even ? t : even > per ? even : per;
  t = t * (wgs <= c.round / 2 ? c.us1 : c.us2) + c.wg * rounds;
  const double mem = kv_bytes / 5e6 * rounds * c.round / wgs;
  return (t > mem ? t : mem) + (n > 1 ? 4 + double(rows) * double(n) * (d + 2) * 8 / 4e6 : 0);
}

struct PagedArgs {
  const char *q, *kn, *vn;  // queries; the call's new rows (NULL: in the cache)
  char* out;
  float* lse;               // natural log; NULL: not asked for
  char *kp, *vp;
  float* wp;                // NULL: no weights
  const int32_t *table, *lens;
  int64_t ks[3], vs[3];     // page, head, row strides in bytes
  int32_t B, Hq, Hkv, G;
  int32_t n_pages, max_pages, shift, cap;  // page_size = 1 << shift; cap = max_pages << shift
  int32_t W, ns;
  float scale;              // tau log2(e): scores in the log2 domain
  int32_t npiece, piece;    // workgroups per row tile, keys of each at least
  float *acc, *ml;          // partial records: acc [row][npiece][d], ml [row][npiece][2]
  float* scores;            // decode with weights: [B][Hq][nv] raw scores (log2 domain)
  float* lse2;              // log2-domain lse by row, where weights need it
  int64_t nv;               // row length of scores
  int32_t per_head;         // decode: table and lens have a row for every (sequence, KV head)
};

// The sequences of one prefill launch (at most kMaxSeqPerLaunch), in the
// kernel arguments.
struct PagedSeqs {
  int32_t nseq, seq0;
  int32_t start[kMaxSeqPerLaunch];     // packed row of the first new token
  int32_t len[kMaxSeqPerLaunch];       // new tokens
  int32_t tile0[kMaxSeqPerLaunch + 1]; // first row tile
};

struct EvictArgs {
  char *kp, *vp;
  float* wp;
  const int32_t *table, *lens, *dst;
  int64_t ks[3], vs[3];
  int32_t B, Hkv, d, esize;
  int32_t n_pages, max_pages, shift, cap;
  int32_t ns, budget, recent;
  int32_t in_place;
  int32_t *kept, *new_lens;
};

// keys: visible tokens of a sequence, at most (it sizes a grid only)
hipError_t launch_paged_decode(const PagedArgs& a, int64_t keys, int d, int dtype, hipStream_t stream);
// tile_rows: kPagedRows (attend_rows), kSharedRows (attend_shared) or kTileRows
// (attend_tiles, bf16 only)
hipError_t launch_paged_prefill(const PagedArgs& a, const PagedSeqs& s, int d, int dtype, int tile_rows,
                                hipStream_t stream);
hipError_t launch_paged_weights(const PagedArgs& a, const PagedSeqs& s, int n_observe, int64_t keys, int d, int dtype,
                                hipStream_t stream);
// Rows row0 .. row0 + rows - 1 of a call in a.npiece > 1 pieces: their records joined.
hipError_t launch_paged_join(const PagedArgs& a, int64_t row0, int64_t rows, int d, int dtype, hipStream_t stream);
hipError_t launch_paged_evict(const EvictArgs& a, hipStream_t stream);

// A row of zeros (device memory): what is read in place of a row that has no
// part in the sums, so that no bits of it reach a product.
static __device__ const uint4 zero_row[32] = {};

// Rows come through global loads.  (A pointer picked from the pools, the
// call's new rows and zero_row is a generic one to the compiler, and generic
// loads count as LDS accesses too: every LDS wait would wait for them.)
typedef const char __attribute__((address_space(1))) * gptr_t;
// NT: non-temporal, for rows that one workgroup reads once (a decode call).
// 32 sequences of 16K..32K tokens (3.2 GB) 577 -> 536 us, and a session of 8K
// (34 MB, in the Infinity Cache from step to step) 18.1 -> 16.8.
template <bool NT>
__device__ __forceinline__ uint4 gload16(gptr_t p) {
  typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
  const auto q = (const u32x4_t __attribute__((address_space(1)))*)p;
  if constexpr (NT) return __builtin_bit_cast(uint4, __builtin_nontemporal_load(q));
  else return __builtin_bit_cast(uint4, *q);
}
// Eight elements.
template <bool NT>
__device__ __forceinline__ void gload_frag(Frag<bf16_t>& f, gptr_t p) { f.v = gload16<NT>(p); }
template <bool NT>
__device__ __forceinline__ void gload_frag(Frag<float>& f, gptr_t p) {
  const float4 a = __builtin_bit_cast(float4, gload16<NT>(p)), b = __builtin_bit_cast(float4, gload16<NT>(p + 16));
  f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
  f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
}

// Page and slot of position j of the sequence whose table row is `row`;
// false where its page is not allocated.
struct Slot {
  int32_t page, slot;
  bool ok;
};
__device__ __forceinline__ Slot paged_slot(const int32_t* row, int32_t j, int32_t shift, int32_t n_pages) {
  Slot s;
  s.page = row[j >> shift];
  s.slot = j & ((1 << shift) - 1);
  s.ok = uint32_t(s.page) < uint32_t(n_pages);
  return s;
}
__device__ __forceinline__ int64_t slot_offset(const int64_t* st, const Slot& s, int g) {
  return int64_t(s.page) * st[0] + int64_t(g) * st[1] + int64_t(s.slot) * st[2];
}

// The tokens that any query at positions t0 .. t1 sees, counted through: the
// sinks before the window, then the window.
struct Seen {
  int32_t sinks, start, n;  // j(v) = v < sinks ? v : v - sinks + start, v in [0, n)
  __device__ __forceinline__ int32_t pos(int32_t v) const { return v < sinks ? v : v - sinks + start; }
};
__device__ __forceinline__ Seen seen_by(int32_t t0, int32_t t1, int32_t W, int32_t ns) {
  Seen s;
  s.start = t0 - W + 1 > 0 ? t0 - W + 1 : 0;
  if (s.start > t1 + 1) s.start = t1 + 1;  // W = 0
  s.sinks = ns < s.start ? ns : s.start;
  s.n = s.sinks + (t1 + 1 - s.start);
  return s;
}

// Inclusive sum over the lanes of a wave: within rows of 16, then the rows'
// last lanes (15 into rows 1 and 3, 31 into rows 2 and 3) to the rows behind.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_add(uint32_t x) {
  return x + uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x = dpp_add<0x111, 0xf>(x);  // row_shr:1
  x = dpp_add<0x112, 0xf>(x);
  x = dpp_add<0x114, 0xf>(x);
  x = dpp_add<0x118, 0xf>(x);
  x = dpp_add<0x142, 0xa>(x);     // row_bcast:15
  return dpp_add<0x143, 0xc>(x);  // row_bcast:31
}

}  // namespace glide
