// Eviction from a paged cache by accumulated attention weight.
#include "paged.h"

namespace glide {

namespace {

__device__ __forceinline__ int32_t seq_len(const EvictArgs& a, int b) {
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : n > a.cap ? a.cap : n;
}

// Weights in order as unsigned numbers: NaN (0) < -inf < ... < -0 = +0 < ... < +inf.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) return 0;
  const uint32_t u = w == 0.f ? 0u : __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int64_t weight_at(const EvictArgs& a, int32_t page, int g, int32_t j) {
  return ((int64_t(page) * a.Hkv + g) << a.shift) + (j & ((1 << a.shift) - 1));
}

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kBins = 2048, kCopies = 2;

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
// Exclusive sum over the workgroup's threads; wsum: one entry per wave.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t* wsum, uint32_t* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint32_t inc = wave_scan(x);
  __syncthreads();
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  // every wave sums the 16 waves' totals in its first row
  const uint32_t w = wave_scan(wsum[lane & (kSelWaves - 1)]);
  const uint32_t before = __builtin_amdgcn_readlane(w, wave ? wave - 1 : 0);
  *total = __builtin_amdgcn_readlane(w, kSelWaves - 1);
  return (wave ? before : 0) + inc - x;
}

// Which tokens stay, one workgroup per (sequence, KV head).  The need-th
// largest key is found by its 11, 11 and 10 bits: a histogram in LDS of the
// keys that agree so far (integer counts, so no order of atomics shows), then
// the bin by a sum from the top.  Then every key above it stays, and the first
// of those equal to it; ranks are counts before a key in the order of
// positions.  Keys are read once and kept in LDS up to KEYS tokens, four
// neighbours to a thread in the passes; longer sequences go through LDS in
// segments, read again per pass.  Bound by the latency of the reads and of two
// dozen barriers, and by the instructions of 16 waves on one CU: 8K tokens 10.7
// us, 16K..32K 27 (256 of them, one per CU), 450..700 7.2.  (Keys in
// registers, their loops unrolled: 24 us at 8K tokens and 21 at 700, most of
// it the fetch of the code.)
template <int KEYS>
__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a) {
  constexpr int QUADS = KEYS / (4 * kSelThreads), NC = QUADS * kSelWaves;  // counts, one per 256 positions
  constexpr int U = QUADS * 4 < 16 ? QUADS * 4 : 16;
  __shared__ uint4 key4[KEYS / 4];
  __shared__ uint32_t hist[kBins * kCopies];
  __shared__ uint32_t cnt[NC];
  __shared__ uint32_t wsum[kSelWaves], pick[2];
  static_assert(NC <= kSelThreads, "a thread per count");
  uint32_t* key = reinterpret_cast<uint32_t*>(key4);
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t len = seq_len(a, b);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  int32_t* kept = a.kept + int64_t(blockIdx.x) * a.budget;
  const int32_t m = len < a.budget ? len : a.budget;
  for (int32_t j = m + tid; j < a.budget; j += kSelThreads) kept[j] = -1;
  if (len <= a.budget) {
    for (int32_t j = tid; j < m; j += kSelThreads) kept[j] = j;
    return;
  }
  // tokens [0, lo) and [hi, len) stay; those between go by their weights
  const int32_t lo = a.ns < len ? a.ns : len;
  const int32_t hi = len - a.recent > lo ? len - a.recent : lo;
  const uint32_t quota = uint32_t(m - lo - (len - hi));
  for (int32_t j = tid; j < lo; j += kSelThreads) kept[j] = j;
  for (int32_t j = tid; j < len - hi; j += kSelThreads) kept[lo + quota + j] = hi + j;
  if (quota == 0) return;

  // Keys of positions [j0, j0 + KEYS) to LDS, up to 16 loads of a thread at
  // once; the quads of a thread that hold any.  Behind the last key zeros, the
  // smallest: at most equal to the threshold, and then behind every real one.
  auto load = [&](int32_t j0) {
    const int32_t n = hi - j0 < KEYS ? hi - j0 : KEYS, quads = (n + 4 * kSelThreads - 1) / (4 * kSelThreads);
    __syncthreads();
    for (int32_t i0 = 0; i0 < quads * 4 * kSelThreads; i0 += U * kSelThreads) {
      int32_t page[U];
      float w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int32_t i = i0 + u * kSelThreads + tid;
        page[u] = i < n ? trow[(j0 + i) >> a.shift] : -1;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int32_t i = i0 + u * kSelThreads + tid;
        w[u] = uint32_t(page[u]) < uint32_t(a.n_pages) ? a.wp[weight_at(a, page[u], g, j0 + i)] : NAN;
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (i0 + u * kSelThreads + tid < KEYS) key[i0 + u * kSelThreads + tid] = weight_key(w[u]);
    }
    __syncthreads();
    return quads;
  };
  const bool once = hi - lo <= KEYS;
  int quads = 0;
  if (once) quads = load(lo);

  uint32_t need = quota, thr = 0;
  int shift = 32;
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass < 2 ? 11 : 10, below = shift;  // bits [below, 32) of thr are known
    shift -= bits;
    for (int i = tid; i < kBins * kCopies; i += kSelThreads) hist[i] = 0;
    __syncthreads();
    for (int32_t j0 = lo; j0 < hi; j0 += KEYS) {
      if (!once) quads = load(j0);
      for (int r = 0; r < quads; ++r) {
        const uint4 k = key4[r * kSelThreads + tid];
        const uint32_t x[4] = {k.x, k.y, k.z, k.w};
        const int32_t left = hi - j0 - (r * kSelThreads + tid) * 4;  // (the zeros behind would all meet in one bin)
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (pass == 0 ? u < left : ((x[u] ^ thr) >> below) == 0)
            atomicAdd(&hist[((x[u] >> shift) & ((1u << bits) - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
      }
    }
    __syncthreads();
    // two bins per thread, from the top: thread t has bins 2047 - 2t, 2046 - 2t
    const uint4 h = reinterpret_cast<const uint4*>(hist)[kBins / 2 - 1 - tid];
    const uint32_t c0 = h.z + h.w, c1 = h.x + h.y;
    uint32_t total;
    const uint32_t above = block_scan(c0 + c1, wsum, &total);
    if (above < need && above + c0 + c1 >= need) {
      const bool second = above + c0 < need;
      pick[0] = kBins - 1 - 2 * tid - (second ? 1 : 0);
      pick[1] = need - above - (second ? c0 : 0);
    }
    __syncthreads();
    thr |= pick[0] << shift;
    need = pick[1];
  }

  // In order: a key above thr stays, and of those equal to it the first
  // `need`, so a kept key's place is the number above before it, and of the
  // equal ones before it at most `need`.  Both counts go through one scan, a
  // half of a word each (up to 32768).
  int32_t above = 0, equal = 0;  // in the segments before
  const int32_t most = int32_t(need);
  for (int32_t j0 = lo; j0 < hi; j0 += KEYS) {
    if (!once) quads = load(j0);
    uint32_t before[QUADS];  // within the wave's 256 positions
    __syncthreads();
#pragma unroll
    for (int r = 0; r < QUADS; ++r) {
      if (r >= quads) continue;
      const uint4 k = key4[r * kSelThreads + tid];
      const uint32_t e = (k.x == thr) + (k.y == thr) + (k.z == thr) + (k.w == thr);
      const uint32_t x = e << 16 | ((k.x > thr) + (k.y > thr) + (k.z > thr) + (k.w > thr));
      const uint32_t inc = wave_scan(x);
      before[r] = inc - x;
      if (lane == 63) cnt[r * kSelWaves + wave] = inc;
    }
    uint32_t all;
    __syncthreads();
    const bool mine = tid < quads * kSelWaves;
    const uint32_t sum = block_scan(mine ? cnt[tid] : 0, wsum, &all);
    if (mine) cnt[tid] = sum;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < QUADS; ++r) {
      if (r >= quads) continue;
      const uint4 k = key4[r * kSelThreads + tid];
      const uint32_t x[4] = {k.x, k.y, k.z, k.w}, c = cnt[r * kSelWaves + wave] + before[r];
      int32_t ne = equal + int32_t(c >> 16), ng = above + int32_t(c & 0xffffu);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const bool gt = x[u] > thr, eq = x[u] == thr;
        if (gt || (eq && ne < most)) kept[lo + ng + (ne < most ? ne : most)] = j0 + (r * kSelThreads + tid) * 4 + u;
        ng += gt;
        ne += eq;
      }
    }
    equal += int32_t(all >> 16);
    above += int32_t(all & 0xffffu);
  }
}

__device__ __forceinline__ Slot slot_of(const EvictArgs& a, const int32_t* row, int32_t j) {
  return paged_slot(row, j, a.shift, a.n_pages);
}

// Kept rows to fresh pages: 32 tokens of a (sequence, KV head) per workgroup,
// every 16-byte piece of K and V on a thread of its own.  Bound by memory: 4096
// tokens of 256 heads, 1.1 GB moved in 216 us (5.0 TB/s).
constexpr int kMoveRows = 32;
__global__ __launch_bounds__(256) void evict_copy(EvictArgs a) {
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int32_t* drow = a.dst + int64_t(b) * a.max_pages;
  const int32_t* kept = a.kept + int64_t(blockIdx.x) * a.budget;
  if (g == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
    const int32_t len = seq_len(a, b);
    a.new_lens[b] = len < a.budget ? len : a.budget;
  }
  const int per = a.d * a.esize / 16, c = (threadIdx.x % per) * 16;  // 8, 16 or 32 pieces of a row
  for (int32_t j0 = blockIdx.y * kMoveRows; j0 < a.budget; j0 += gridDim.y * kMoveRows) {
    const int32_t jend = j0 + kMoveRows < a.budget ? j0 + kMoveRows : a.budget;
    for (int32_t j = j0 + threadIdx.x / per; j < jend; j += 256 / per) {
      const int32_t src = kept[j];
      if (src < 0) continue;
      const Slot s = slot_of(a, trow, src), t = slot_of(a, drow, j);
      uint4 k = make_uint4(0, 0, 0, 0), v = k;
      float w = 0.f;
      if (s.ok) {
        k = *reinterpret_cast<const uint4*>(a.kp + slot_offset(a.ks, s, g) + c);
        v = *reinterpret_cast<const uint4*>(a.vp + slot_offset(a.vs, s, g) + c);
        if (c == 0) w = a.wp[weight_at(a, s.page, g, src)];
      }
      if (t.ok) {
        *reinterpret_cast<uint4*>(a.kp + slot_offset(a.ks, t, g) + c) = k;
        *reinterpret_cast<uint4*>(a.vp + slot_offset(a.vs, t, g) + c) = v;
        if (c == 0) a.wp[weight_at(a, t.page, g, j)] = w;
      }
    }
  }
}

// Kept rows to their places in the same pages.  Tokens move towards the front
// and stay in order, so a row read in a step (all of its rows before any is
// written) is never behind a row written in a step before: one barrier per
// step of up to 1024 rows.  A workgroup moves 128 bytes of every K, or V, row
// of a (sequence, KV head), or its weights.  32 sequences of 16K..32K tokens to
// 4096 (8 heads of 128, bf16) 230 us = 4.7 TB/s; one of 32K to 16K 102 us (1.3
// TB/s): the chain kept -> table -> row -> barrier of 40 workgroups.
__global__ __launch_bounds__(1024) void evict_move(EvictArgs a) {
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv;
  const int slabs = a.d * a.esize / 128, what = blockIdx.y / slabs;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int32_t* kept = a.kept + int64_t(blockIdx.x) * a.budget;
  if (what == 2) {
    if (g == 0 && threadIdx.x == 0) {
      const int32_t len = seq_len(a, b);
      a.new_lens[b] = len < a.budget ? len : a.budget;
    }
    for (int32_t j0 = 0; j0 < a.budget; j0 += 1024) {
      const int32_t j = j0 + threadIdx.x, src = j < a.budget ? kept[j] : -1;
      float w = 0.f;
      if (src > j) {
        const Slot s = slot_of(a, trow, src);
        if (s.ok) w = a.wp[weight_at(a, s.page, g, src)];
      }
      __syncthreads();
      if (src > j) {
        const Slot t = slot_of(a, trow, j);
        if (t.ok) a.wp[weight_at(a, t.page, g, j)] = w;
      }
    }
    return;
  }
  char* pool = what ? a.vp : a.kp;
  const int64_t* st = what ? a.vs : a.ks;
  const int c = int(blockIdx.y % slabs) * 128 + (threadIdx.x & 7) * 16;
  constexpr int N = 8;  // rows of a thread per step
  for (int32_t j0 = 0; j0 < a.budget; j0 += 128 * N) {
    if (kept[j0] < 0) break;  // (kept is -1 from its last entry on)
    int32_t src[N];
    uint4 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int32_t j = j0 + 128 * i + (threadIdx.x >> 3);
      src[i] = j < a.budget ? kept[j] : -1;
      if (src[i] <= j) src[i] = -1;  // in its place already
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      x[i] = make_uint4(0, 0, 0, 0);
      if (src[i] < 0) continue;
      const Slot s = slot_of(a, trow, src[i]);
      if (s.ok) x[i] = *reinterpret_cast<const uint4*>(pool + slot_offset(st, s, g) + c);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (src[i] < 0) continue;
      const Slot t = slot_of(a, trow, j0 + 128 * i + (threadIdx.x >> 3));
      if (t.ok) *reinterpret_cast<uint4*>(pool + slot_offset(st, t, g) + c) = x[i];
    }
  }
}

}  // namespace

hipError_t launch_paged_evict(const EvictArgs& a, hipStream_t stream) {
  const uint32_t units = uint32_t(a.B) * a.Hkv;
  // the smaller LDS lets a CU hold several of them
  if (a.cap <= 4096) evict_select<4096><<<units, kSelThreads, 0, stream>>>(a);
  else evict_select<32768><<<units, kSelThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.in_place) {
    evict_move<<<dim3(units, 2 * uint32_t(a.d * a.esize / 128) + 1), 1024, 0, stream>>>(a);
  } else {
    const int64_t n = (int64_t(a.budget) + kMoveRows - 1) / kMoveRows;
    evict_copy<<<dim3(units, uint32_t(n < 65535 ? n : 65535)), 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

}  // namespace glide
