// The pages that a query attends to: a score of every page from the element-wise
// bounds of its keys, and the largest scores of each query and KV head.
#include <algorithm>

#include "select.h"

namespace glide {

namespace {

__device__ __forceinline__ int32_t seq_len(const SelectArgs& a, int b) {
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : n > a.cap ? a.cap : n;
}
// A score as a number that orders alike; NaN below all others.  0 is kept for
// pages that cannot be selected, all ones for those that always are.
__device__ __forceinline__ uint64_t key_of(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  if (x != x) return 1;
  return (u >> 63) ? ~u : u | (uint64_t(1) << 63);
}
constexpr uint64_t kAlways = ~uint64_t(0);

template <typename T>
__device__ __forceinline__ void load8d(double* x, const char* p) {
  Frag<T> f;
  gload_frag<false>(f, (gptr_t)p);
  float y[8];
  f.to_floats(y);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = double(y[i]);
}

// ---------------------------------------------------------------------------
// Scores of pages: with u_c = sum_h max(q_hc, 0) and w_c = sum_h min(q_hc, 0)
// over the group's heads, sum_c (u_c kmax_c + w_c kmin_c) is no less than
// sum_h q_h . k of any key of the page, for two products of a row instead of G
// per key.  In fp64, where products of bf16 numbers are exact: neighbouring
// pages' scores are told apart alike however the sum is ordered.
// D / 8 lanes to a page, eight elements of both bounds each, for up to eight
// queries of a sequence; bound by the reading of the bounds.
template <typename T, int D>
__global__ __launch_bounds__(256) void page_scores(SelectArgs a, PagedSeqs s) {
  constexpr int SL = D / 8, ES = int(sizeof(T)), PPI = 256 / SL;  // lanes of a page, pages at once
  __shared__ __align__(16) double uw[kScoreRows][2][D];
  const int tile = int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  int lo = 0, hi = s.nseq - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.tile0[mid] <= tile) lo = mid;
    else hi = mid - 1;
  }
  const int b = s.seq0 + lo, ntok = s.len[lo];
  const int32_t begin = s.start[lo] > a.row0 ? s.start[lo] : a.row0;
  const int32_t end = s.start[lo] + ntok < a.row1 ? s.start[lo] + ntok : a.row1;
  const int32_t r0 = begin + (tile - s.tile0[lo]) * kScoreRows;
  const int rows = end - r0 < kScoreRows ? end - r0 : kScoreRows;
  const int32_t len = seq_len(a, b), t0 = len - ntok + (r0 - s.start[lo]);  // position of the first row
  const int32_t last = t0 + rows - 1 < 0 ? -1 : (t0 + rows - 1) >> a.shift;
  if (int(blockIdx.y) * kScorePages > last) return;
  for (int e = threadIdx.x; e < rows * D; e += 256) {
    const T* q = reinterpret_cast<const T*>(a.q) + (int64_t(r0 + e / D) * a.Hq + g * a.G) * D + e % D;
    double u = 0, w = 0;
    for (int h = 0; h < a.G; ++h) {
      const float x = a.negative ? -to_f32(q[h * D]) : to_f32(q[h * D]);
      u += x < 0.f ? 0.f : x;   // (NaN counts in u: the score is NaN)
      w += x < 0.f ? x : 0.f;
    }
    uw[e / D][0][e % D] = w;
    uw[e / D][1][e % D] = u;
  }
  __syncthreads();
  const int sub = threadIdx.x % SL;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  for (int32_t i0 = blockIdx.y * kScorePages; i0 <= last; i0 += gridDim.y * kScorePages) {
#pragma unroll 1
    for (int32_t i = i0 + int32_t(threadIdx.x) / SL; i < i0 + kScorePages; i += PPI) {
      if (i > last) break;
      const int32_t page = trow[i];
      const bool ok = uint32_t(page) < uint32_t(a.n_pages);
      double kmin[8], kmax[8];
      const char* p = a.bounds + (int64_t(ok ? page : 0) * a.Hkv + g) * (2 * D * ES) + sub * 8 * ES;
      load8d<T>(kmin, p);
      load8d<T>(kmax, p + D * ES);
      for (int r = 0; r < rows; ++r) {
        double x = 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) x = fma(uw[r][1][8 * sub + c], kmax[c], fma(uw[r][0][8 * sub + c], kmin[c], x));
#pragma unroll
        for (int m = 1; m < SL; m *= 2) x += __shfl_xor(x, m);
        const int32_t mine = (t0 + r) >> a.shift;  // (t0 + r < 0: behind no page)
        if (sub == 0 && i <= mine) {
          uint64_t k = key_of(x);
          if (i < a.n_first || i > mine - a.n_recent) k = kAlways;
          a.keys[(int64_t(r0 - a.row0 + r) * a.Hkv + g) * a.max_pages + i] = ok ? k : 0;
        }
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The n_select largest keys of a row, in the order of their pages; of equal
// ones the first.  The least key that is in is found from the highest bit in
// which keys differ down, 11 bits at a time: a histogram of the keys that agree
// so far, and its bins from the top.  KEYS: keys of a thread in registers; 0:
// read again in each pass.
template <int KEYS>
__global__ __launch_bounds__(256) void select_pages(SelectArgs a, PagedSeqs s) {
  constexpr int BITS = 11, BINS = 1 << BITS, PER = BINS / 256;
  __shared__ uint32_t hist[BINS];
  __shared__ uint64_t red[2][4];
  __shared__ uint32_t cnt[3][4], found[3], ranks[(KEYS ? KEYS : 1) * 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t row = a.row0 + int32_t(blockIdx.x) / a.Hkv;
  const int g = int(blockIdx.x) % a.Hkv;
  int lo = 0, hi = s.nseq - 1;
  while (lo < hi) {  // the last sequence that starts at or before the row
    const int mid = (lo + hi + 1) >> 1;
    if (s.start[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  const int b = s.seq0 + lo;
  const int32_t t = seq_len(a, b) - s.len[lo] + (row - s.start[lo]);
  const int32_t n = t < 0 ? 0 : (t >> a.shift) + 1;  // pages up to the row's
  const int64_t unit = int64_t(row - a.row0) * a.Hkv + g;
  const uint64_t* keys = a.keys + unit * a.max_pages;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  int32_t* out = a.selected + (int64_t(row) * a.Hkv + g) * a.n_select;
  int32_t* pages = a.pages + unit * a.n_select;

  uint64_t mine[KEYS ? KEYS : 1];
  if constexpr (KEYS > 0) {
#pragma unroll
    for (int e = 0; e < KEYS; ++e) {
      const int32_t i = e * 256 + int32_t(threadIdx.x);
      mine[e] = i < n ? keys[i] : 0;
    }
  }
  auto each = [&](auto f) {
    if constexpr (KEYS > 0) {
#pragma unroll
      for (int e = 0; e < KEYS; ++e) f(mine[e]);
    } else {
      for (int32_t i = threadIdx.x; i < n; i += 256) f(keys[i]);
    }
  };
  // sums and extremes over the workgroup
  uint32_t always = 0, free_ = 0;
  uint64_t top = 0, bottom = ~uint64_t(0);
  each([&](uint64_t k) {
    if (k == kAlways) ++always;
    else if (k) {
      ++free_;
      top = k > top ? k : top;
      bottom = k < bottom ? k : bottom;
    }
  });
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    always += __shfl_xor(always, m);
    free_ += __shfl_xor(free_, m);
    const uint64_t x = __shfl_xor((unsigned long long)top, m), y = __shfl_xor((unsigned long long)bottom, m);
    top = x > top ? x : top;
    bottom = y < bottom ? y : bottom;
  }
  if (lane == 0) {
    cnt[0][wave] = always;
    cnt[1][wave] = free_;
    red[0][wave] = top;
    red[1][wave] = bottom;
  }
  __syncthreads();
  always = free_ = 0;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    always += cnt[0][w];
    free_ += cnt[1][w];
    top = red[0][w] > top ? red[0][w] : top;
    bottom = red[1][w] < bottom ? red[1][w] : bottom;
  }
  uint32_t want = always < uint32_t(a.n_select) ? uint32_t(a.n_select) - always : 0;
  const uint32_t count = want < free_ ? always + want : always + free_;
  // in: keys at or above `least` (among equals of it the first `ties`, where that is not all of them)
  uint64_t least = 1;
  uint32_t ties = ~0u;
  if (want == 0) {
    least = kAlways;
  } else if (want < free_) {
    int shift = 64 - __builtin_clzll((top ^ bottom) | 1);  // bits below it differ
    uint64_t prefix = shift < 64 ? top >> shift : 0;         // of the keys that agree so far
    for (;;) {
      const int step = shift < BITS ? shift : BITS, next = shift - step;
#pragma unroll
      for (int i = 0; i < PER; ++i) hist[i * 256 + threadIdx.x] = 0;
      __syncthreads();
      each([&](uint64_t k) {
        if (k && k != kAlways && (shift < 64 ? k >> shift : 0) == prefix)
          atomicAdd(&hist[(k >> next) & ((uint64_t(1) << step) - 1)], 1u);
      });
      __syncthreads();
      // bins from the top: thread x has bins BINS - 1 - PER x downwards
      uint32_t h[PER], sum = 0;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        h[i] = hist[BINS - 1 - int(threadIdx.x) * PER - i];
        sum += h[i];
      }
      uint32_t upto = sum;
#pragma unroll
      for (int m = 1; m < 64; m *= 2) {
        const uint32_t y = __shfl_up(upto, m);
        upto += lane >= m ? y : 0;
      }
      if (lane == 63) cnt[2][wave] = upto;
      __syncthreads();
      for (int w = 0; w < wave; ++w) upto += cnt[2][w];
      uint32_t above = upto - sum;
      if (above < want && upto >= want) {  // one thread: the bin that the last one in is in
        bool done = false;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (!done && above + h[i] >= want) {
            found[0] = BINS - 1 - threadIdx.x * PER - i;
            found[1] = above;
            found[2] = h[i];
            done = true;
          }
          if (!done) above += h[i];
        }
      }
      __syncthreads();
      const uint32_t bin = found[0];
      want -= found[1];
      prefix = (prefix << step) | bin;
      shift = next;
      if (found[2] == want || shift == 0) {
        if (found[2] != want) ties = want;
        least = prefix << shift;
        break;
      }
    }
  }
  // ranks of the pages that are in
  auto emit = [&](int32_t i, uint32_t at) {
    out[at] = i;
    pages[at] = trow[i];
  };
  auto place = [&](auto in, auto put) {  // in(k, i): counted; put(i, rank)
    if constexpr (KEYS > 0) {
      uint64_t mask[KEYS];
#pragma unroll
      for (int e = 0; e < KEYS; ++e) {
        mask[e] = __ballot(in(mine[e]));
        if (lane == 0) ranks[e * 4 + wave] = __popcll(mask[e]);
      }
      __syncthreads();
      uint32_t before = 0;
      for (int x = 0; x < wave; ++x) before += ranks[x];
#pragma unroll
      for (int e = 0; e < KEYS; ++e) {
        if ((mask[e] >> lane) & 1)
          put(e, e * 256 + int32_t(threadIdx.x), before + __popcll(mask[e] & ((uint64_t(1) << lane) - 1)));
        if (e + 1 < KEYS)
          for (int x = 0; x < 4; ++x) before += ranks[e * 4 + wave + x];
      }
      __syncthreads();
    } else {
      uint32_t before = 0;
      for (int32_t i0 = 0; i0 < n; i0 += 256) {
        const int32_t i = i0 + int32_t(threadIdx.x);
        const uint64_t m = __ballot(i < n && in(i < n ? keys[i] : 0));
        if (lane == 0) ranks[wave] = __popcll(m);
        __syncthreads();
        uint32_t at = before;
        for (int x = 0; x < wave; ++x) at += ranks[x];
        if ((m >> lane) & 1) put(0, i, at + __popcll(m & ((uint64_t(1) << lane) - 1)));
        for (int x = 0; x < 4; ++x) before += ranks[x];
        __syncthreads();
      }
    }
  };
  if (ties == ~0u) {
    place([&](uint64_t k) { return k >= least && k; }, [&](int, int32_t i, uint32_t at) { emit(i, at); });
  } else {
    // equal keys: the first `ties` of them
    if constexpr (KEYS > 0) {
      place([&](uint64_t k) { return k == least; }, [&](int e, int32_t, uint32_t at) {
#pragma unroll
        for (int x = 0; x < KEYS; ++x)
          if (x == e && at >= ties) mine[x] = 0;
      });
      place([&](uint64_t k) { return k >= least; }, [&](int, int32_t i, uint32_t at) { emit(i, at); });
    } else {
      uint32_t before = 0, equal = 0;
      for (int32_t i0 = 0; i0 < n; i0 += 256) {
        const int32_t i = i0 + int32_t(threadIdx.x);
        const uint64_t k = i < n ? keys[i] : 0;
        const uint64_t e = __ballot(k == least);
        if (lane == 0) ranks[wave] = __popcll(e);
        __syncthreads();
        uint32_t at = equal;
        for (int x = 0; x < wave; ++x) at += ranks[x];
        at += __popcll(e & ((uint64_t(1) << lane) - 1));
        for (int x = 0; x < 4; ++x) equal += ranks[x];
        const bool in = k > least || (k == least && at < ties);
        __syncthreads();
        const uint64_t m = __ballot(in);
        if (lane == 0) ranks[wave] = __popcll(m);
        __syncthreads();
        at = before;
        for (int x = 0; x < wave; ++x) at += ranks[x];
        if (in) emit(i, at + __popcll(m & ((uint64_t(1) << lane) - 1)));
        for (int x = 0; x < 4; ++x) before += ranks[x];
        __syncthreads();
      }
    }
  }
  for (uint32_t i = count + threadIdx.x; i < uint32_t(a.n_select); i += 256) {
    out[i] = -1;
    pages[i] = -1;
  }
  // tokens of the selected pages that the row sees: the last page may be its own
  if (threadIdx.x == 0) {
    const bool own = n > 0 && uint32_t(trow[n - 1]) < uint32_t(a.n_pages);  // (its own is always in)
    a.held[unit] = count == 0 ? 0 : int32_t((count << a.shift) - (own ? (uint32_t(n) << a.shift) - 1 - t : 0));
  }
}

template <typename T, int D>
hipError_t scores_t(const SelectArgs& a, const PagedSeqs& s, int64_t pages, hipStream_t stream) {
  const dim3 grid(uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv),
                  uint32_t(std::max<int64_t>(1, std::min<int64_t>((pages + kScorePages - 1) / kScorePages, 4096))));
  page_scores<T, D><<<grid, 256, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_select(const SelectArgs& a, const PagedSeqs& s, int64_t pages, int d, int dtype,
                         hipStream_t stream) {
  const hipError_t e =
      dtype == GLIDE_BF16
          ? (d == 128 ? scores_t<bf16_t, 128>(a, s, pages, stream) : scores_t<bf16_t, 64>(a, s, pages, stream))
          : (d == 128 ? scores_t<float, 128>(a, s, pages, stream) : scores_t<float, 64>(a, s, pages, stream));
  if (e != hipSuccess) return e;
  const uint32_t units = uint32_t(a.row1 - a.row0) * uint32_t(a.Hkv);
  // (by the table's width, which no sequence has more pages than)
  if (a.max_pages <= 1024) select_pages<4><<<units, 256, 0, stream>>>(a, s);
  else if (a.max_pages <= 4096) select_pages<16><<<units, 256, 0, stream>>>(a, s);
  else select_pages<0><<<units, 256, 0, stream>>>(a, s);
  return hipGetLastError();
}

}  // namespace glide
