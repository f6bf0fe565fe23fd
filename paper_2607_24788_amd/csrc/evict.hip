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

__device__ __forceinline__ uint32_t key_at(const EvictArgs& a, const int32_t* trow, int g, int32_t j) {
  const Slot s = paged_slot(trow, j, a.shift, a.n_pages);
  return s.ok ? weight_key(a.wp[((int64_t(s.page) * a.Hkv + g) << a.shift) + s.slot]) : 0u;
}

constexpr int kSelThreads = 1024;

// Exclusive sum over the workgroup of a flag, and its total.
__device__ __forceinline__ int block_rank(bool flag, int* wsum, int* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const uint64_t m = __ballot(flag);
  __syncthreads();
  if (lane == 0) wsum[wave] = __popcll(m);
  __syncthreads();
  int before = 0, all = 0;
  for (int w = 0; w < kSelThreads / 64; ++w) {
    if (w < wave) before += wsum[w];
    all += wsum[w];
  }
  *total = all;
  return before + __popcll(m & ((uint64_t(1) << lane) - 1));
}

// Which tokens stay, one workgroup per (sequence, KV head): the need-th
// largest key by four passes over its bytes (histograms in LDS, integer
// counts: no order of atomics shows), then the kept positions in order.
__global__ __launch_bounds__(kSelThreads) void evict_select(EvictArgs a) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t pick[2];
  __shared__ int wsum[kSelThreads / 64];
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, tid = threadIdx.x;
  const int32_t len = seq_len(a, b);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  int32_t* kept = a.kept + int64_t(blockIdx.x) * a.budget;
  const int32_t m = len < a.budget ? len : a.budget;
  for (int32_t j = m + tid; j < a.budget; j += kSelThreads) kept[j] = -1;
  if (len <= a.budget) {
    for (int32_t j = tid; j < m; j += kSelThreads) kept[j] = j;
    return;
  }
  const int32_t lo = a.ns < len ? a.ns : len;
  const int32_t hi = len - a.recent > lo ? len - a.recent : lo;
  uint32_t need = uint32_t(m - lo - (len - hi)), thr = 0xffffffffu;
  if (need > 0) {
    thr = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) hist[tid] = 0;
      __syncthreads();
      const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
      for (int32_t j = lo + tid; j < hi; j += kSelThreads) {
        const uint32_t k = key_at(a, trow, g, j);
        if ((k & mask) == thr) atomicAdd(&hist[(k >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint32_t left = need;
        int bin = 255;
        while (hist[bin] < left) left -= hist[bin--];
        pick[0] = bin;
        pick[1] = left;
      }
      __syncthreads();
      thr |= pick[0] << shift;
      need = pick[1];
    }
  }
  // in order: every key above thr, and the first `need` of those equal to it
  int32_t at = 0, equal = 0;
  for (int32_t j0 = 0; j0 < len; j0 += kSelThreads) {
    const int32_t j = j0 + tid;
    bool keep = j < len && (j < lo || j >= hi);
    const uint32_t k = j >= lo && j < hi ? key_at(a, trow, g, j) : 0u;
    const bool eq = j >= lo && j < hi && k == thr;
    int total;
    const int before = block_rank(eq, wsum, &total);
    keep = keep || (j >= lo && j < hi && (k > thr || (eq && uint32_t(equal + before) < need)));
    equal += total;
    const int rank = block_rank(keep, wsum, &total);
    if (keep) kept[at + rank] = j;
    at += total;
  }
}

// Kept rows to their places.  Tokens move towards the front and stay in
// order, so a tile's rows, read before any of them is written, are never
// behind a row written before: in place needs one barrier per tile.
__global__ __launch_bounds__(1024) void evict_move(EvictArgs a) {
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, what = blockIdx.y;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int32_t* drow = a.dst + int64_t(b) * a.max_pages;
  const int32_t* kept = a.kept + int64_t(blockIdx.x) * a.budget;
  if (what == 2) {
    if (g == 0 && threadIdx.x == 0) {
      const int32_t len = seq_len(a, b);
      a.new_lens[b] = len < a.budget ? len : a.budget;
    }
    for (int32_t j0 = 0; j0 < a.budget; j0 += 1024) {
      const int32_t j = j0 + threadIdx.x, src = j < a.budget ? kept[j] : -1;
      float w = 0.f;
      if (src >= 0) {
        const Slot s = paged_slot(trow, src, a.shift, a.n_pages);
        if (s.ok) w = a.wp[((int64_t(s.page) * a.Hkv + g) << a.shift) + s.slot];
      }
      __syncthreads();
      if (src >= 0) {
        const Slot s = paged_slot(drow, j, a.shift, a.n_pages);
        if (s.ok) a.wp[((int64_t(s.page) * a.Hkv + g) << a.shift) + s.slot] = w;
      }
    }
    return;
  }
  char* pool = what ? a.vp : a.kp;
  const int64_t* st = what ? a.vs : a.ks;
  const int per = a.d * a.esize / 16, rows = 1024 / per;  // 16-byte pieces of a row, rows at a time
  const int c = (threadIdx.x % per) * 16;
  for (int32_t j0 = 0; j0 < a.budget; j0 += rows) {
    const int32_t j = j0 + threadIdx.x / per, src = j < a.budget ? kept[j] : -1;
    uint4 x = make_uint4(0, 0, 0, 0);
    if (src >= 0) {
      const Slot s = paged_slot(trow, src, a.shift, a.n_pages);
      if (s.ok) x = *reinterpret_cast<const uint4*>(pool + slot_offset(st, s, g) + c);
    }
    __syncthreads();
    if (src >= 0) {
      const Slot s = paged_slot(drow, j, a.shift, a.n_pages);
      if (s.ok) *reinterpret_cast<uint4*>(pool + slot_offset(st, s, g) + c) = x;
    }
  }
}

}  // namespace

hipError_t launch_paged_evict(const EvictArgs& a, hipStream_t stream) {
  const uint32_t units = uint32_t(a.B) * a.Hkv;
  evict_select<<<units, kSelThreads, 0, stream>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  evict_move<<<dim3(units, 3), 1024, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace glide
