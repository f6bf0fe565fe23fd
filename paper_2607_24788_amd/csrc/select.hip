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

__device__ __forceinline__ void load4(float* x, const float* p) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void load4(float* x, const bf16_t* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  x[0] = __uint_as_float(v.x << 16);
  x[1] = __uint_as_float(v.x & 0xffff0000u);
  x[2] = __uint_as_float(v.y << 16);
  x[3] = __uint_as_float(v.y & 0xffff0000u);
}

// Sum over SL lanes (8, or a row of 16), in each of them, in one order.
template <int CTRL>
__device__ __forceinline__ double dpp_mv64(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(u)), CTRL, 0xf, 0xf, false));
  const uint32_t hi = uint32_t(__builtin_amdgcn_update_dpp(0, int(uint32_t(u >> 32)), CTRL, 0xf, 0xf, false));
  return __builtin_bit_cast(double, uint64_t(hi) << 32 | lo);
}
template <int SL>
__device__ __forceinline__ double sum_lanes(double x) {
  static_assert(SL == 8 || SL == 16, "half a row, or a row");
  x += dpp_mv64<0xb1>(x);   // quad_perm [1,0,3,2]
  x += dpp_mv64<0x4e>(x);   // quad_perm [2,3,0,1]
  x += dpp_mv64<0x141>(x);  // row_half_mirror
  if constexpr (SL == 16) x += dpp_mv64<0x140>(x);  // row_mirror
  return x;
}

// ---------------------------------------------------------------------------
// Scores of pages: with u_c = sum_h max(q_hc, 0) and w_c = sum_h min(q_hc, 0)
// over the group's heads, sum_c (u_c kmax_c + w_c kmin_c) is no less than
// sum_h q_h . k of any key of the page, for two products of a row instead of G
// per key.  In fp64, summed in one order: pages of the same bounds have the same
// score, and others are told apart down to that sum's rounding.
// D / 8 lanes to a page, eight elements of both bounds each (asked for a page
// ahead), for up to eight queries of a sequence.
template <typename T, int D>
__global__ __launch_bounds__(256) void page_scores(SelectArgs a, PagedSeqs s) {
  constexpr int SL = D / 8, ES = int(sizeof(T)), PPI = 256 / SL;  // lanes of a page, pages at once
  __shared__ __align__(16) double uw[kScoreRows][2][D];
  const int tile = int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  int lo = a.single ? tile : 0, hi = a.single ? tile : s.nseq - 1;
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
  if (int(blockIdx.y) * a.chunk > last) return;
  const int sub = threadIdx.x % SL;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  struct Page {
    Frag<T> lo, hi;
    bool ok;
  };
  auto fetch = [&](int32_t i) {
    Page p;
    const int32_t page = trow[i < last ? i : last];
    p.ok = uint32_t(page) < uint32_t(a.n_pages);
    const gptr_t at = (gptr_t)a.bounds + (int64_t(p.ok ? page : 0) * a.Hkv + g) * (2 * D * ES) + sub * 8 * ES;
    if (a.single) {  // read once: 32 sequences of 769 pages, 80.5 -> 77.8 us of the call
      gload_frag<true>(p.lo, at);
      gload_frag<true>(p.hi, at + D * ES);
    } else {
      gload_frag<false>(p.lo, at);
      gload_frag<false>(p.hi, at + D * ES);
    }
    return p;
  };
  // pages of this workgroup: a.chunk in turn with the others
  const int32_t mine = int32_t(threadIdx.x) / SL, jump = (int32_t(gridDim.y) - 1) * a.chunk;
  int32_t i0 = int32_t(blockIdx.y) * a.chunk, in = 0;
  Page next = fetch(i0 + mine);
  // four elements of a row to a thread, four heads' at once
  static_assert(kScoreRows * D / 4 <= 256, "a thread for each");
  if (int(threadIdx.x) < rows * (D / 4)) {
    const int r = threadIdx.x / (D / 4), c0 = (threadIdx.x % (D / 4)) * 4;
    const T* q = reinterpret_cast<const T*>(a.q) + (int64_t(r0 + r) * a.Hq + g * a.G) * D + c0;
    double u[4] = {}, w[4] = {};
    for (int h0 = 0; h0 < a.G; h0 += 4) {
      float x[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) load4(x[k], q + (h0 + k < a.G ? h0 + k : h0) * D);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (h0 + k >= a.G) break;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const float y = a.negative ? -x[k][c] : x[k][c];
          u[c] += y < 0.f ? 0.f : y;  // (NaN counts in u: the score is NaN)
          w[c] += y < 0.f ? y : 0.f;
        }
      }
    }
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      uw[r][0][c0 + c] = w[c];
      uw[r][1][c0 + c] = u[c];
    }
  }
  __syncthreads();
  while (i0 <= last) {
    const Page now = next;
    const int32_t i = i0 + mine;
    in += PPI;
    i0 += PPI;
    if (in >= a.chunk) {
      in = 0;
      i0 += jump;
    }
    if (i0 <= last) next = fetch(i0 + mine);
    double kmin[8], kmax[8];
    float y[8];
    now.lo.to_floats(y);
#pragma unroll
    for (int c = 0; c < 8; ++c) kmin[c] = double(y[c]);
    now.hi.to_floats(y);
#pragma unroll
    for (int c = 0; c < 8; ++c) kmax[c] = double(y[c]);
#pragma unroll 2
    for (int r = 0; r < rows; ++r) {
      double x = 0, z = 0;
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        x = fma(uw[r][1][8 * sub + c], kmax[c], x);
        z = fma(uw[r][0][8 * sub + c], kmin[c], z);
      }
      x = sum_lanes<SL>(x + z);
      const int32_t own = (t0 + r) >> a.shift;  // (t0 + r < 0: behind no page)
      if (sub == 0 && i <= own) {
        uint64_t k = key_of(x);
        if (i < a.n_first || i > own - a.n_recent) k = kAlways;
        a.keys[(int64_t(r0 - a.row0 + r) * a.Hkv + g) * a.max_pages + i] = now.ok ? k : 0;
      }
    }
  }
}

// ---------------------------------------------------------------------------
// The n_select largest keys of a row, in the order of their pages; of equal
// ones the first.  The least key that is in is found from the highest bit in
// which keys differ down, 11 bits at a time: a histogram in LDS of the keys that
// agree so far (integer counts: no order of atomics shows), and its bins from
// the top; two or three of these, as the bin of the last key in has few others.
// Then ranks by one scan.  Four neighbouring pages to a thread; ONE: all of them
// at once, in registers, else in turns, read again in each pass.
// Bound by the latency of its reads and barriers.
template <int NT, bool ONE>
__global__ __launch_bounds__(NT) void select_pages(SelectArgs a, PagedSeqs s) {
  constexpr int BITS = 11, BINS = 1 << BITS, PER = BINS / NT, NW = NT / 64;
  __shared__ uint32_t hist[BINS], wsum[NW], total[4], found[3];  // total: always in, others, and their extremes
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t row = a.row0 + int32_t(blockIdx.x) / a.Hkv;
  const int g = int(blockIdx.x) % a.Hkv;
  int lo = a.single ? row - a.row0 : 0, hi = a.single ? lo : s.nseq - 1;
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

  uint64_t mine[4];
  auto load = [&](int32_t i0) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int32_t i = i0 + 4 * int32_t(threadIdx.x) + e;
      mine[e] = i < n ? keys[i] : 0;
    }
  };
  auto each = [&](auto f) {
    if constexpr (ONE) {
#pragma unroll
      for (int e = 0; e < 4; ++e) f(mine[e]);
    } else {
      for (int32_t i0 = 0; i0 < n; i0 += 4 * NT) {
        load(i0);
#pragma unroll
        for (int e = 0; e < 4; ++e) f(mine[e]);
      }
    }
  };
  // exclusive sum over the workgroup's threads, and the sum of all
  auto block_scan = [&](uint32_t x, uint32_t* all) {
    const uint32_t inc = wave_scan(x);
    __syncthreads();
    if (lane == 63) wsum[wave] = inc;
    __syncthreads();
    const uint32_t w = wave_scan(lane < NW ? wsum[lane] : 0);
    *all = __builtin_amdgcn_readlane(w, 63);
    return (wave ? __builtin_amdgcn_readlane(w, wave - 1) : 0) + inc - x;
  };
  if constexpr (ONE) load(0);
  if (threadIdx.x < 4) total[threadIdx.x] = threadIdx.x == 3 ? ~0u : 0u;
#pragma unroll
  for (int i = 0; i < PER; ++i) hist[i * NT + threadIdx.x] = 0;
  __syncthreads();
  uint32_t always = 0, others = 0, top = 0, bottom = ~0u;  // extremes: upper halves
  each([&](uint64_t k) {
    const bool other = k != 0 && k != kAlways;
    always += __popcll(__ballot(k == kAlways));
    others += __popcll(__ballot(other));
    const uint32_t h = uint32_t(k >> 32);
    top = other && h > top ? h : top;
    bottom = other && h < bottom ? h : bottom;
  });
#pragma unroll
  for (int m = 1; m < 64; m *= 2) {
    const uint32_t x = uint32_t(__shfl_xor(int(top), m)), y = uint32_t(__shfl_xor(int(bottom), m));
    top = x > top ? x : top;
    bottom = y < bottom ? y : bottom;
  }
  if (lane == 0) {
    atomicAdd(&total[0], always);
    atomicAdd(&total[1], others);
    atomicMax(&total[2], top);
    atomicMin(&total[3], bottom);
  }
  __syncthreads();
  always = total[0];
  others = total[1];
  top = total[2];
  bottom = total[3];
  uint32_t want = always < uint32_t(a.n_select) ? uint32_t(a.n_select) - always : 0;
  const uint32_t count = want < others ? always + want : always + others;
  // in: keys above `least`, and the first `ties` of those equal to it
  uint64_t least = want == 0 ? kAlways - 1 : 0;
  uint32_t ties = 0;
  if (want != 0 && want < others) {
    int shift = top == bottom ? 32 : 64 - __builtin_clz(top ^ bottom);  // bits below it differ
    uint64_t prefix = shift < 64 ? uint64_t(top) << 32 >> shift : 0;    // of the keys that agree so far
    for (;;) {
      const int step = shift < BITS ? shift : BITS, next = shift - step;
      each([&](uint64_t k) {
        if (k && k != kAlways && (shift < 64 ? k >> shift : 0) == prefix)
          atomicAdd(&hist[(k >> next) & ((uint64_t(1) << step) - 1)], 1u);
      });
      __syncthreads();
      // bins from the top: thread x has bins BINS - 1 - PER x downwards
      uint32_t h[PER], sum = 0, all;
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        h[i] = hist[BINS - 1 - int(threadIdx.x) * PER - i];
        sum += h[i];
      }
      uint32_t above = block_scan(sum, &all);
      if (above < want && above + sum >= want) {  // one thread: the bin that the last one in is in
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
#pragma unroll
      for (int i = 0; i < PER; ++i) hist[BINS - 1 - int(threadIdx.x) * PER - i] = 0;
      __syncthreads();
      want -= found[1];
      prefix = (prefix << step) | found[0];
      shift = next;
      if (found[2] == want) {
        least = (prefix << shift) - 1;  // (no key but one that cannot be selected is 0)
        break;
      }
      if (shift == 0) {
        least = prefix;
        ties = want;
        break;
      }
    }
  }
  // ranks, in the order of pages: counts of both kinds in one scan (4096 at most)
  uint32_t above = 0, equal = 0;
  for (int32_t i0 = 0; i0 < n; i0 += 4 * NT) {
    if constexpr (!ONE) load(i0);
    uint32_t x = 0, all;
#pragma unroll
    for (int e = 0; e < 4; ++e) x += (mine[e] > least ? 1u : 0u) + (ties && mine[e] == least ? 1u << 16 : 0u);
    const uint32_t before = block_scan(x, &all);
    uint32_t up = above + (before & 0xffffu), eq = equal + (before >> 16);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int32_t i = i0 + 4 * int32_t(threadIdx.x) + e;
      const bool is = ties && mine[e] == least, in = mine[e] > least || (is && eq < ties);
      if (in) {
        const uint32_t at = up + (eq < ties ? eq : ties);
        out[at] = i;
        pages[at] = trow[i];
      }
      up += mine[e] > least;
      eq += is;
    }
    above += all & 0xffffu;
    equal += all >> 16;
  }
  for (uint32_t i = count + threadIdx.x; i < uint32_t(a.n_select); i += NT) {
    out[i] = -1;
    pages[i] = -1;
  }
  // tokens of the selected pages that the row sees: the last page may be its own
  if (threadIdx.x == 0) {
    const bool own = n > 0 && uint32_t(trow[n - 1]) < uint32_t(a.n_pages);  // (its own is always in)
    a.held[unit] = count == 0 ? 0 : int32_t((count << a.shift) - (own ? (uint32_t(n) << a.shift) - 1 - t : 0));
  }
}

// ---------------------------------------------------------------------------
// Attention of many (row, KV head) units over their selected pages, a wave to a
// unit: the products and the way through LDS of a tile of 32 keys are those of
// attend_rows, whose four waves share a unit; without their join, and with eight
// units to a CU instead of two, it goes further where units are many.  Bound by
// the caches: neighbouring rows' pages are the same or other ones.
// a.table and a.lens have a row for every unit; every page in it is allocated.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void picked_rows(PagedArgs a, int32_t units) {
  constexpr int KK = D / 32, CT = D / 16, ES = int(sizeof(T)), TK = 32;
  constexpr bool KLDS = ES == 2;
  constexpr int RS = D + (KLDS ? 16 : 4), LPR = D * ES / 16, RPI = 64 / LPR, NL = TK / RPI;
  __shared__ __align__(16) T klds[KLDS ? 4 : 1][KLDS ? TK * RS : 1];
  __shared__ __align__(16) T vlds[4][TK * RS];
  const int lane = threadIdx.x & 63, n = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t unit = int32_t(blockIdx.x) * 4 + wave;
  if (unit >= units) return;
  const int g = unit % a.Hkv;
  const int32_t held = __builtin_amdgcn_readfirstlane(a.lens[unit]);
  const int32_t* trow = a.table + int64_t(unit) * a.max_pages;
  const bool rok = n < a.G;
  const int64_t orow = int64_t(unit / a.Hkv) * a.Hq + g * a.G + (rok ? n : 0);
  Frag<T> qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    qf[kk].load(reinterpret_cast<const T*>(a.q) + orow * D + 32 * kk + 8 * lg);
    if (!rok) qf[kk].zero();
    if (a.scale < 0) qf[kk].negate();  // scores of -q: the frame is a maximum of raw scores
  }
  const float c = fabsf(a.scale);
  float m = kNoMax, l = 0.f;
  f32x4_t acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = zero4();
  T *kt = klds[KLDS ? wave : 0], *vt = vlds[wave];

  // rows of a tile: lane x looks up key x % 32 a tile ahead; rows behind the last are zeros
  auto look = [&](int32_t x) {
    const int32_t v = x + (lane & 31);
    return v < held ? trow[v >> a.shift] : -1;
  };
  Frag<T> kf[2][KK], vf[2][KK];  // bf16: NL pieces each
  auto fetch = [&](int32_t x, int32_t page) {
#pragma unroll
    for (int e = 0; e < (KLDS ? NL : 2); ++e) {
      const int row = KLDS ? e * RPI + lane / LPR : 16 * e + n;
      const int32_t p = __shfl(page, row);
      const Slot sl = {p, (x + row) & ((1 << a.shift) - 1), true};
      const gptr_t kr = p >= 0 ? (gptr_t)a.kp + slot_offset(a.ks, sl, g) : (gptr_t)zero_row;
      const gptr_t vr = p >= 0 ? (gptr_t)a.vp + slot_offset(a.vs, sl, g) : (gptr_t)zero_row;
      if constexpr (KLDS) {
        gload_frag<false>(kf[e / KK][e % KK], kr + (lane % LPR) * 16);
        gload_frag<false>(vf[e / KK][e % KK], vr + (lane % LPR) * 16);
      } else {
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) gload_frag<false>(kf[e][kk], kr + (32 * kk + 8 * lg) * ES);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) gload_frag<false>(vf[e][kk], vr + (32 * kk + 8 * lg) * ES);
      }
    }
  };
  int32_t page = 0;
  if (held > 0) {
    const int32_t first = look(0);
    page = look(TK);
    fetch(0, first);
  }
  for (int32_t x = 0; x < held; x += TK) {
    f32x4_t sc[2] = {zero4(), zero4()};
    if constexpr (KLDS) {
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        const int at = (e * RPI + lane / LPR) * RS + (lane % LPR) * 8;
        *reinterpret_cast<uint4*>(kt + at) = kf[e / KK][e % KK].v;
        *reinterpret_cast<uint4*>(vt + at) = vf[e / KK][e % KK].v;
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          sc[t] = mma(kf[t][kk], qf[kk], sc[t]);
          float w[8];
          vf[t][kk].to_floats(w);
          float4* at = reinterpret_cast<float4*>(vt + (16 * t + n) * RS + 32 * kk + 8 * lg);
          at[0] = make_float4(w[0], w[1], w[2], w[3]);
          at[1] = make_float4(w[4], w[5], w[6], w[7]);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (x + TK < held) {
      const int32_t now = page;
      page = look(x + 2 * TK);
      fetch(x + TK, now);
    }
    if constexpr (KLDS) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          Frag<T> k;
          k.load(kt + (16 * t + n) * RS + 32 * kk + 8 * lg);
          sc[t] = mma(k, qf[kk], sc[t]);
        }
    }
    if (held - x < TK) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (x + 16 * t + 4 * lg + i >= held) sc[t][i] = -INFINITY;
    }
    // the frame moves only when a score passes it by 2^8: weights up to that
    // round alike, and fp32 sums hold them
    float mx = sc[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[t][i]);
    mx = lg_max(mx) * c;
    if (__any(mx > m + 8.f)) {
      const float m2 = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[ct][i] *= f;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], c, -m));
      l += p[i];
    }
    Frag<T> pf;
    pf.set8(p);  // bf16: weights rounded to half a step, 2^-8 of each at most
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      Frag<T> vc;
      load_colfrag2(vc, vt, RS, 4 * lg, 16 + 4 * lg, 16 * ct);
      acc[ct] = mma(vc, pf, acc[ct]);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  l = lg_sum(l);
  if (!rok) return;
  if (lg == 0 && a.lse) a.lse[orow] = (l > 0.f ? m + __builtin_amdgcn_logf(l) : l == 0.f ? -INFINITY : l) * kLn2;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* w = reinterpret_cast<T*>(a.out) + orow * D + 4 * lg;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float y[4] = {acc[ct][0] * inv, acc[ct][1] * inv, acc[ct][2] * inv, acc[ct][3] * inv};
    if constexpr (ES == 2)
      *reinterpret_cast<uint2*>(w + 16 * ct) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
    else
      *reinterpret_cast<float4*>(w + 16 * ct) = make_float4(y[0], y[1], y[2], y[3]);
  }
}

// ---------------------------------------------------------------------------
// The same (bf16) for neighbouring rows of a sequence together: a wave takes R = 16 / G
// rows of one KV head, whose heads fill the MFMA's columns, over the pages that
// any of them selects, in order; a page that several rows select is read once.
// The rows' lists are merged on the way: 64 / R lanes hold the next entries of
// each, a step takes the least head of all.  A tile of 32 keys lies in one page;
// of a page of 16 it has the 16.
//   A value that is not finite would reach every column (0 times infinity): in a
//   tile that some row does not see in full such values are looked for, and where
//   there are any the rows take the tile one by one, each with the rows of V that
//   it sees and the others 0.
struct Picked {
  const int32_t* selected;
  int32_t n_select, row0, row1;  // the launch's rows
  int32_t R, lanes;              // rows of a wave, log2 of the lanes of each row's list
  int32_t units;
};
template <int D>
__global__ __launch_bounds__(256, 2) void picked_tiles(PagedArgs a, PagedSeqs s, Picked w) {
  typedef bf16_t T;
  constexpr int KK = D / 32, CT = D / 16, TK = kTileSlots, RS = D + 16, LPR = D / 8, RPI = 64 / LPR, NL = TK / RPI;
  __shared__ __align__(16) T klds[4][TK * RS], vlds[4][TK * RS];
  const int lane = threadIdx.x & 63, n = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t unit = int32_t(blockIdx.x) * 4 + wave;
  if (unit >= w.units) return;
  const int tile = unit / a.Hkv, g = unit % a.Hkv;
  int si = 0, hi = s.nseq - 1;
  while (si < hi) {
    const int mid = (si + hi + 1) >> 1;
    if (s.tile0[mid] <= tile) si = mid;
    else hi = mid - 1;
  }
  const int b = s.seq0 + si, ntok = s.len[si];
  const int32_t begin = s.start[si] > w.row0 ? s.start[si] : w.row0;
  const int32_t end = s.start[si] + ntok < w.row1 ? s.start[si] + ntok : w.row1;
  const int32_t r0 = begin + (tile - s.tile0[si]) * w.R;
  const int rows = end - r0 < w.R ? end - r0 : w.R;
  int32_t len = a.lens[b];
  len = __builtin_amdgcn_readfirstlane(len < 0 ? 0 : len > a.cap ? a.cap : len);
  const int32_t t0 = len - ntok + (r0 - s.start[si]), tmax = t0 + rows - 1;  // positions of the first row and the last
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const bool rok = n < rows * a.G;
  const int rr = rok ? n / a.G : rows - 1;  // this lane's row
  const int32_t tr = t0 + rr;
  const int64_t orow = int64_t(r0 - w.row0 + rr) * a.Hq + g * a.G + (rok ? n - rr * a.G : 0);
  Frag<T> qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    qf[kk].load(reinterpret_cast<const T*>(a.q) + orow * D + 32 * kk + 8 * lg);
    if (!rok) qf[kk].zero();
    if (a.scale < 0) qf[kk].negate();  // scores of -q: the frame is a maximum of raw scores
  }
  const float c = fabsf(a.scale);
  float m = kNoMax, l = 0.f;
  f32x4_t acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = zero4();
  T *kt = klds[wave], *vt = vlds[wave];

  // the rows' lists: lane (row, x) has entry x of the row's current run and of the next
  const int LW = 1 << w.lanes, lrow = lane >> w.lanes, lx = lane & (LW - 1);
  const int32_t* list = w.selected + (int64_t(r0 + (lrow < rows ? lrow : 0)) * a.Hkv + g) * w.n_select;
  auto run = [&](int32_t at) { return lrow < rows && at + lx < w.n_select ? list[at + lx] : -1; };
  int32_t idx = 0, cur = run(0), nxt = run(LW);
  struct Tile {
    int32_t j0, page;  // first position, page in the pools
    uint64_t rows;     // at lane (row, 0): whether the row selects the page
  };
  auto next_page = [&]() {
    int32_t h = __shfl(cur, (lane & ~(LW - 1)) + (idx & (LW - 1)));
    if (h < 0) h = kNoTile;
    int32_t least = h;
    for (int x = LW; x < 64; x *= 2) {
      const int32_t y = __shfl_xor(least, x);
      least = y < least ? y : least;
    }
    least = __builtin_amdgcn_readfirstlane(least);
    Tile t = {kNoTile, 0, __ballot(h == least)};
    if (least == kNoTile) return t;
    if (h == least) {
      ++idx;
      if ((idx & (LW - 1)) == 0) {
        cur = nxt;
        nxt = run(idx + LW);
      }
    }
    t.j0 = least << a.shift;
    t.page = trow[least];
    return t;
  };
  auto next_tile = [&](Tile t) {
    t.j0 = next_in_page(t.j0, a.shift, tmax);
    return t.j0 != kNoTile ? t : next_page();
  };
  Frag<T> kf[NL], vf[NL];  // whole rows by neighbouring lanes
  const int32_t keys = a.shift < 5 ? 1 << a.shift : TK;  // of a tile
  auto fetch = [&](const Tile& t) {
    const int32_t page = __builtin_amdgcn_readfirstlane(t.page), slot = t.j0 & ((1 << a.shift) - 1);
    const gptr_t kb = (gptr_t)a.kp + slot_offset(a.ks, Slot{page, slot, true}, g);
    const gptr_t vb = (gptr_t)a.vp + slot_offset(a.vs, Slot{page, slot, true}, g);
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int row = e * RPI + lane / LPR;
      const bool there = row < keys && t.j0 + row <= tmax;  // (rows behind the last query are zeros)
      gload_frag<false>(kf[e], (there ? kb + int64_t(row) * a.ks[2] : (gptr_t)zero_row) + (lane % LPR) * 16);
      gload_frag<false>(vf[e], (there ? vb + int64_t(row) * a.vs[2] : (gptr_t)zero_row) + (lane % LPR) * 16);
    }
  };
  // whether the fetched tile has values that are not finite: an exponent of ones carries into the bit above it
  auto nonfinite = [&]() {
    uint32_t x = 0;
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const uint4 v = vf[e].v;
      x |= ((v.x & 0x7f807f80u) + 0x00800080u) | ((v.y & 0x7f807f80u) + 0x00800080u) |
           ((v.z & 0x7f807f80u) + 0x00800080u) | ((v.w & 0x7f807f80u) + 0x00800080u);
    }
    x &= 0x80008000u;
    return __any(x != 0);
  };
  auto order = [] {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  uint64_t every = 0;  // of Tile::rows: all rows
  for (int x = 0; x < rows; ++x) every |= (LW == 64 ? ~uint64_t(0) : ((uint64_t(1) << LW) - 1) << (x * LW));

  Tile now = next_page();
  if (now.j0 != kNoTile) fetch(now);
  Tile after = next_tile(now);
  while (now.j0 != kNoTile) {
    const int32_t j0 = now.j0;
    const uint64_t mine = now.rows;
    // (a tile that all rows see in full needs no mask)
    const bool full = keys == TK && (mine & every) == every && j0 + TK - 1 <= t0;
    const bool bad = !full && nonfinite();
    f32x4_t sc[2] = {zero4(), zero4()};
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int at = (e * RPI + lane / LPR) * RS + (lane % LPR) * 8;
      *reinterpret_cast<uint4*>(kt + at) = kf[e].v;
      *reinterpret_cast<uint4*>(vt + at) = vf[e].v;
    }
    order();
    now = after;
    if (now.j0 != kNoTile) {
      fetch(now);
      after = next_tile(now);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        Frag<T> k;
        k.load(kt + (16 * t + n) * RS + 32 * kk + 8 * lg);
        sc[t] = mma(k, qf[kk], sc[t]);
      }
    if (!full) {
      const bool sees = rok && ((mine >> (rr << w.lanes)) & 1);
      const int32_t most = sees ? (tr - j0 < keys ? tr - j0 : keys - 1) - 4 * lg : -1;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (16 * t + i > most) sc[t][i] = -INFINITY;
    }
    // the frame moves only when a score passes it by 2^8: weights up to that
    // round alike, and fp32 sums hold them
    float mx = sc[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, sc[t][i]);
    mx = lg_max(mx) * c;
    if (__any(mx > m + 8.f)) {
      const float m2 = fmaxf(m, mx), f = __builtin_amdgcn_exp2f(m - m2);
      m = m2;
      l *= f;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[ct][i] *= f;
    }
    float p[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], c, -m));
      l += p[i];
    }
    Frag<T> pf;
    pf.set8(p);  // bf16: weights rounded to half a step, 2^-8 of each at most
    if (!bad) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        Frag<T> vc;
        load_colfrag2(vc, vt, RS, 4 * lg, 16 + 4 * lg, 16 * ct);
        acc[ct] = mma(vc, pf, acc[ct]);
      }
    } else {
      // from the last row back: each sees no more than the one after it
#pragma unroll 1
      for (int x = rows - 1; x >= 0; --x) {
        if (!((mine >> (x << w.lanes)) & 1)) continue;
        const int32_t keep = t0 + x - j0 + 1;  // keys of the tile that it sees
        order();
#pragma unroll 1
        for (int key = keep > 0 ? keep : 0; key < TK; ++key)
          for (int e = lane; e < D; e += 64) vt[key * RS + e] = T(0);
        order();
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          Frag<T> vc;
          load_colfrag2(vc, vt, RS, 4 * lg, 16 + 4 * lg, 16 * ct);
          const f32x4_t y = mma(vc, pf, zero4());
#pragma unroll
          for (int i = 0; i < 4; ++i) acc[ct][i] += rr == x ? y[i] : 0.f;
        }
      }
    }
    order();
  }
  l = lg_sum(l);
  if (!rok) return;
  if (lg == 0 && a.lse) a.lse[orow] = (l > 0.f ? m + __builtin_amdgcn_logf(l) : l == 0.f ? -INFINITY : l) * kLn2;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  T* o = reinterpret_cast<T*>(a.out) + orow * D + 4 * lg;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float y[4] = {acc[ct][0] * inv, acc[ct][1] * inv, acc[ct][2] * inv, acc[ct][3] * inv};
    *reinterpret_cast<uint2*>(o + 16 * ct) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
  }
}

template <typename T, int D>
hipError_t scores_t(const SelectArgs& a, const PagedSeqs& s, int64_t pages, hipStream_t stream) {
  const dim3 grid(uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv),
                  uint32_t(std::max<int64_t>(1, std::min<int64_t>((pages + a.chunk - 1) / a.chunk, 32768))));
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
  if (a.max_pages <= 1024) select_pages<256, true><<<units, 256, 0, stream>>>(a, s);
  else if (a.max_pages <= 4096) select_pages<1024, true><<<units, 1024, 0, stream>>>(a, s);
  else select_pages<1024, false><<<units, 1024, 0, stream>>>(a, s);
  return hipGetLastError();
}

hipError_t launch_picked_tiles(const PagedArgs& a, const PagedSeqs& s, const SelectArgs& e, int rows, int d,
                               hipStream_t stream) {
  int lanes = 6;
  while ((64 >> lanes) < rows) --lanes;
  const Picked w = {e.selected, e.n_select, e.row0, e.row1, rows, lanes, s.tile0[s.nseq] * a.Hkv};
  const uint32_t n = (uint32_t(w.units) + 3) / 4;
  if (d == 128) picked_tiles<128><<<n, 256, 0, stream>>>(a, s, w);
  else picked_tiles<64><<<n, 256, 0, stream>>>(a, s, w);
  return hipGetLastError();
}

hipError_t launch_picked(const PagedArgs& a, int32_t units, int d, int dtype, hipStream_t stream) {
  const uint32_t n = (uint32_t(units) + 3) / 4;
  if (dtype == GLIDE_BF16) {
    if (d == 128) picked_rows<bf16_t, 128><<<n, 256, 0, stream>>>(a, units);
    else picked_rows<bf16_t, 64><<<n, 256, 0, stream>>>(a, units);
  } else {
    if (d == 128) picked_rows<float, 128><<<n, 256, 0, stream>>>(a, units);
    else picked_rows<float, 64><<<n, 256, 0, stream>>>(a, units);
  }
  return hipGetLastError();
}

}  // namespace glide
