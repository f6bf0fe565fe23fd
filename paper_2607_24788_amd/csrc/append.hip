// New rows into a paged cache, rotated on the way; the element-wise bounds of a
// page's keys; rows of a 4-bit cache read back.
#include <algorithm>

#include "append.h"

namespace glide {

namespace {

__device__ __forceinline__ int find_seq(const PagedSeqs& s, int tile) {
  int lo = 0, hi = s.nseq - 1;  // the last sequence whose first tile is <= tile
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (s.tile0[mid] <= tile) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ int32_t seq_len(const int32_t* lens, int b, int32_t cap) {
  const int32_t n = lens[b];
  return n < 0 ? 0 : n > cap ? cap : n;
}

template <typename T>
__device__ __forceinline__ void load8(float* x, const char* p) {
  Frag<T> f;
  gload_frag<false>(f, (gptr_t)p);
  f.to_floats(x);
}
template <typename T>
__device__ __forceinline__ void store8(char* p, const float* x) {
  if constexpr (sizeof(T) == 2) {
    Frag<T> f;
    f.set8(x);
    *reinterpret_cast<uint4*>(p) = f.v;
  } else {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
}
// Sine and cosine of t turns, |t| <= 1/2, in fp64: the nearest quarter off, then
// their series up to x^15 / 15! and x^16 / 16!, x at most pi / 4 (what follows is
// 6e-17 of x at most).  The coefficients come from memory: it is called seldom,
// and they would take registers all along.
__constant__ const double kSeries[8][2] = {
    {-1. / 1307674368000, 1. / 20922789888000}, {1. / 6227020800, -1. / 87178291200},
    {-1. / 39916800, 1. / 479001600},           {1. / 362880, -1. / 3628800},
    {-1. / 5040, 1. / 40320},                   {1. / 120, -1. / 720},
    {-1. / 6, 1. / 24},                         {1., -0.5}};
constexpr double kTurn = 0.15915494309189533577;  // 1 / (2 pi)
__device__ __forceinline__ void sincos_turn(double t, double* sn, double* cs) {
  const double k = __builtin_rint(4 * t), x = (t - 0.25 * k) * 6.28318530717958647693, z = x * x;
  double s = 0, c = 0;
#pragma unroll 1
  for (int i = 0; i < 8; ++i) {
    s = fma(s, z, kSeries[i][0]);
    c = fma(c, z, kSeries[i][1]);
  }
  s *= x;
  c = fma(c, z, 1.);
  const int q = int(k);
  const double u = q & 1 ? c : s, v = q & 1 ? s : c;
  *sn = q & 2 ? -u : u;
  *cs = (q + 1) & 2 ? -v : v;
}
// Element e of a key, rotated in fp64; row: the key, at: its position.
template <typename T, bool INTER>
__device__ __forceinline__ double rotated(const T* row, int e, const float* freqs, int rot, double at) {
  if (e >= rot) return to_f32(row[e]);
  const int half = rot / 2, p = INTER ? e >> 1 : e < half ? e : e - half;
  const bool second = INTER ? e & 1 : e >= half;
  const double u = to_f32(row[INTER ? 2 * p : p]), v = to_f32(row[INTER ? 2 * p + 1 : p + half]);
  double t = at * (double(freqs[p]) * kTurn), s, c;
  t -= __builtin_rint(t);
  sincos_turn(t, &s, &c);
  return second ? fma(v, c, u * s) : fma(u, c, -(v * s));
}
// The next fp32 number from x >= 0 on, for the scale that it takes: scales end at fp32 numbers.
__device__ __forceinline__ float above(double x) {
  const float y = float(x);
  return double(y) < x ? __uint_as_float(__float_as_uint(y) + 1) : y;
}
__device__ __forceinline__ float group_max(float m) {  // over four neighbouring threads
  m = fmaxf(m, dpp_mv<0xb1, 0xf>(m));
  return fmaxf(m, dpp_mv<0x4e, 0xf>(m));
}
template <typename T>
__device__ __forceinline__ float held(float x) { return to_f32(from_f32<T>(x)); }

// Least and largest of a page's keys, element by element; NaN is left out.
struct Bounds16 {
  float lo[16], hi[16];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      lo[i] = INFINITY;
      hi[i] = -INFINITY;
    }
  }
  __device__ __forceinline__ void add(int i, float x) {
    lo[i] = fminf(lo[i], x);
    hi[i] = fmaxf(hi[i], x);
  }
};
// What a page's bounds are already, of a thread's elements.
template <typename T>
struct OldBounds {
  Frag<T> lo[2], hi[2];
  __device__ __forceinline__ void load(const char* row, int D, int c1, int c2) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const gptr_t p = (gptr_t)row + (h ? c2 : c1) * 8 * int(sizeof(T));
      gload_frag<false>(lo[h], p);
      gload_frag<false>(hi[h], p + D * int(sizeof(T)));
    }
  }
};
// A thread's bounds to the page's row, together with those there if `more`.
template <typename T, int D>
__device__ __forceinline__ void store_bounds(Bounds16& b, const OldBounds<T>& old, char* row, int c1, int c2,
                                             bool more) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    if (more) {
      float lo[8], hi[8];
      old.lo[h].to_floats(lo);
      old.hi[h].to_floats(hi);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        b.lo[8 * h + i] = fminf(b.lo[8 * h + i], lo[i]);
        b.hi[8 * h + i] = fmaxf(b.hi[8 * h + i], hi[i]);
      }
    }
    char* p = row + (h ? c2 : c1) * 8 * int(sizeof(T));
    store8<T>(p, b.lo + 8 * h);
    store8<T>(p + D * sizeof(T), b.hi + 8 * h);
  }
}
// The threads' bounds joined in threads x < C (elements 8 c1 .. and 8 c2 ..; the
// others of a workgroup hold other tokens of the same elements).
template <int C>
__device__ __forceinline__ void join_bounds(Bounds16& b, float (*red)[32]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int m = C; m < 64; m *= 2)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      b.lo[i] = fminf(b.lo[i], __shfl_xor(b.lo[i], m));
      b.hi[i] = fmaxf(b.hi[i], __shfl_xor(b.hi[i], m));
    }
  if (lane < C) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      red[wave * C + lane][i] = b.lo[i];
      red[wave * C + lane][16 + i] = b.hi[i];
    }
  }
  __syncthreads();
  if (int(threadIdx.x) < C) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
      for (int w = 1; w < 4; ++w) {
        b.lo[i] = fminf(b.lo[i], red[w * C + lane][i]);
        b.hi[i] = fmaxf(b.hi[i], red[w * C + lane][16 + i]);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// Appends with rotation.  A workgroup takes the new tokens of one sequence in
// one unit of positions (a page where bounds are kept, so that it alone writes
// them) and, of one KV head, their key, their value and the group's queries: an
// angle's sine and cosine serve G + 1 rows.  A thread has 16 elements of a row
// (half-split pairs: eight and their partners; interleaved: whole pairs), so
// every row is read and written once, in 16-byte pieces.
//   Angles: position times frequency in fp64, as turns; the nearest whole turn
//   is taken off there, and what is left (at most half a turn) goes to fp32:
//   at position 2^20 the angle is off by 2^-25 of a turn, as at position 1.
//   4 bits: a code is that of the key rotated in 64 bits.  Few elements come so
//   near to a step's middle that fp32 could miss it; those alone are worked out
//   in fp64 (8191 tokens and their read back, builds on one card: 56.6 us, in fp32
//   alone 54.3, all of them in fp64 78).
// Bound by HBM in prompts: 8191 tokens of 32 / 8 heads of 128, bf16, with bounds,
// 202 MB in 46 us (4.4 TB/s; from memory.  Rows are read past the caches: 49 us
// through them), 36 out of the caches; into 4 bits 177 MB in 48 (3.7 TB/s) and 33:
// its 122 registers leave four waves to a SIMD, each with a row ahead.  One
// token of 32 sequences takes 6.1 us, of one fp32 layer 4.6: lens -> table ->
// bounds, rows and angles.
// SINGLE: a call of one token per sequence.
template <typename T, int D, bool FOUR, bool INTER, bool SINGLE>
__global__ __launch_bounds__(256) void append_rotated(AppendArgs a, PagedSeqs s) {
  constexpr int C = D / 16, ES = int(sizeof(T)), RB = D * ES, LANES = 256 / C;
  __shared__ float red[FOUR ? 1 : 4 * C][32];
  const int tile = int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  const int si = SINGLE ? tile : find_seq(s, tile), b = s.seq0 + si, ntok = SINGLE ? 1 : s.len[si];
  const int64_t tok0 = SINGLE ? s.start[0] + si : s.start[si];
  const int32_t len = seq_len(a.lens, b, a.cap), p0 = len - ntok;
  const int32_t u0 = ((p0 >> a.unit) + (SINGLE ? 0 : tile - s.tile0[si])) << a.unit;
  const int32_t j0 = p0 > u0 ? p0 : u0, j1 = len - u0 < (1 << a.unit) ? len : u0 + (1 << a.unit);
  const int n = j1 - j0;
  if (n <= 0) return;
  // lanes over rows where there are few tokens
  int RL = 1;
  while (RL < 8 && n * RL * 2 <= LANES) RL *= 2;
  const int c = threadIdx.x % C, x = threadIdx.x / C, rl = x & (RL - 1);
  // the thread's pieces of a row, and whether they are rotated
  int c1 = c, c2 = c + C;
  bool r1, r2;
  if (INTER) {
    r1 = 8 * c1 < a.rot;
    r2 = 8 * c2 < a.rot;
  } else {
    const int half = a.rot / 16;
    r1 = r2 = c < half;
    c1 = r1 ? c : a.rot / 8 + c - half;
    c2 = r1 ? c + half : c1 + (D - a.rot) / 16;
  }
  double f[8];  // turns per position
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int at = INTER ? (i < 4 ? 4 * c1 + i : 4 * c2 + i - 4) : 8 * c1 + i;
    const bool on = INTER ? (i < 4 ? r1 : r2) : r1;
    f[i] = on ? double(a.freqs[at]) * kTurn : 0.0;
  }
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  Bounds16 bd;
  OldBounds<T> old;
  if constexpr (!FOUR) bd.clear();
  // row 0: the key, 1: the value, then the group's queries
  const int nrow = a.q ? a.G + 2 : 2;
  auto row_at = [&](int row, int64_t tok) {
    return row < 2 ? (row == 0 ? a.k : a.v) + (tok * a.Hkv + g) * RB
                   : a.q + (tok * a.Hq + g * a.G + row - 2) * RB;
  };
  for (int32_t j = j0 + x / RL; j < j1; j += LANES / RL) {
    const int64_t tok = tok0 + (j - p0);
    // the first row is asked for before its angles are worked out, the next ones
    // a row ahead (but where the bounds' registers would leave three waves to a
    // SIMD for four: 8191 tokens 47 us with it, 38 without)
    constexpr bool AHEAD = SINGLE || FOUR;
    Frag<T> w1, w2;
    auto fetch = [&](int row) {
      const gptr_t p = (gptr_t)row_at(row, tok);
      gload_frag<true>(w1, p + c1 * 8 * ES);
      gload_frag<true>(w2, p + c2 * 8 * ES);
    };
    if (AHEAD && rl < nrow) fetch(rl);
    Slot sl = {0, 0, false};
    if (j >= 0) sl = paged_slot(trow, j, a.shift, a.n_pages);
    if constexpr (SINGLE && !FOUR) {
      if (a.bounds && int(threadIdx.x) < C && sl.ok && sl.slot > 0)
        old.load(a.bounds + (int64_t(sl.page) * a.Hkv + g) * (2 * RB), D, c1, c2);
    }
    float sn[8], cs[8];
    if (r1 || r2) {
      const double at = a.pos ? a.pos[tok] : j;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        double t = at * f[i];
        t -= __builtin_rint(t);
        sincospif(2.f * float(t), &sn[i], &cs[i]);
      }
    }
    for (int row = rl; row < nrow; row += RL) {
      float y[16];
      if (!AHEAD) fetch(row);
      w1.to_floats(y);
      w2.to_floats(y + 8);
      if (AHEAD && row + RL < nrow) fetch(row + RL);
      if (row < 2 && !sl.ok) continue;
      float size[2] = {0.f, 0.f};  // 4 bits: of a half's pairs |x| + |y| at most, where they are rotated
      if (row != 1) {
        if constexpr (FOUR) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float z = INTER ? fabsf(y[2 * i]) + fabsf(y[2 * i + 1]) : fabsf(y[i]) + fabsf(y[8 + i]);
            const int h = INTER ? i / 4 : 0;
            size[h] = z > size[h] ? z : size[h];
          }
          if (!INTER) size[1] = size[0];
          if (row != 0 || !r1) size[0] = 0.f;
          if (row != 0 || !r2) size[1] = 0.f;
        }
        if constexpr (INTER) {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (i < 4 ? r1 : r2) {
              const float u = y[2 * i], v = y[2 * i + 1];
              y[2 * i] = fmaf(u, cs[i], -(v * sn[i]));
              y[2 * i + 1] = fmaf(v, cs[i], u * sn[i]);
            }
        } else if (r1) {
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float u = y[i], v = y[8 + i];
            y[i] = fmaf(u, cs[i], -(v * sn[i]));
            y[8 + i] = fmaf(v, cs[i], u * sn[i]);
          }
        }
      }
      if (row >= 2) {
        char* to = a.qo + (tok * a.Hq + g * a.G + row - 2) * RB;
        store8<T>(to + c1 * 8 * ES, y);
        store8<T>(to + c2 * 8 * ES, y + 8);
      } else if constexpr (FOUR) {
        // groups of 32 elements: those of four neighbouring threads
        const int64_t at = ((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot;
        uint8_t* codes = (row == 0 ? a.p4.kc : a.p4.vc) + at * (D / 2);
        uint8_t* scales = (row == 0 ? a.p4.ks : a.p4.vs) + at * (D / kGroup4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int ch = h ? c2 : c1;
          float m = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            float& z = y[8 * h + i];
            z = z == z ? z : 0.f;
            m = fmaxf(m, fabsf(z));
          }
          m = group_max(m);
          // What fp32 may be off by, at most: 2^-21 of |x| + |y| (angle 3.2, sine and
          // cosine 2, products and sum 2 half steps), and as much again.  Where that
          // leaves the scale or a code open, the elements are rotated in fp64: about
          // one key in 400.
          const float slack = group_max(size[h]) * 0x1p-20f;
          auto exact = [&](int i) {
            const double z = rotated<T, INTER>(reinterpret_cast<const T*>(row_at(0, tok)), 8 * ch + i, a.freqs, a.rot,
                                               a.pos ? a.pos[tok] : j);
            return z == z ? z : 0.0;
          };
          const bool open = scale_byte(m - slack) != scale_byte(m + slack) && slack > 0.f;
          if (__any(open)) {
            double most = 0;
            if (open) {
#pragma unroll 1
              for (int i = 0; i < 8; ++i) most = fmax(most, fabs(exact(i)));
            }
            const float x = group_max(above(most));
            m = open ? x : m;
          }
          const uint32_t byte = scale_byte(m);
          const float inv = __uint_as_float((254u - byte) << 23);
          float off;
          uint32_t w = codes8(y + 8 * h, inv, &off);
          const float near = 0.5f - 2.f * slack * inv;  // (steps of 1/2 at least)
          if (__any(slack > 0.f && !(off < near))) {
            uint32_t left = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              code_of(fabsf(y[8 * h + i]) * inv, &off);
              left |= off < near ? 0u : 1u << i;
            }
            if (!(slack > 0.f)) left = 0;
#pragma unroll 1
            while (left) {
              const int i = __builtin_ctz(left);
              left &= left - 1;
              const double z = exact(i);
              double rest;
              const uint32_t code = code_of(fabs(z) * double(inv), &rest) | (z < 0 ? 8u : 0u);
              w = (w & ~(15u << (4 * i))) | code << (4 * i);
            }
          }
          *reinterpret_cast<uint32_t*>(codes + ch * 4) = w;
          if ((c & 3) == 0) scales[ch / 4] = uint8_t(byte);
        }
      } else {
        char* to = (row == 0 ? a.kp + slot_offset(a.ks, sl, g) : a.vp + slot_offset(a.vs, sl, g));
        store8<T>(to + c1 * 8 * ES, y);
        store8<T>(to + c2 * 8 * ES, y + 8);
        if (row == 0) {
          if (a.wp && c == 0) a.wp[((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot] = 0.f;
          if (a.bounds) {
#pragma unroll
            for (int i = 0; i < 16; ++i) bd.add(i, held<T>(y[i]));
          }
        }
      }
    }
    if (SINGLE) break;
  }
  if constexpr (!FOUR) {
    if (a.bounds) {
      // (with bounds a unit is a page)
      const int32_t first = j0 > 0 ? j0 : 0;
      if (j1 <= first) return;
      const Slot sl = paged_slot(trow, first, a.shift, a.n_pages);
      if (!sl.ok) return;
      char* row = a.bounds + (int64_t(sl.page) * a.Hkv + g) * (2 * RB);
      if constexpr (!SINGLE) {  // (one token: its key is in threads x < C, and what was there asked for before)
        join_bounds<C>(bd, red);
        if (int(threadIdx.x) < C && sl.slot > 0) old.load(row, D, c1, c2);
      }
      if (int(threadIdx.x) < C) store_bounds<T, D>(bd, old, row, c1, c2, sl.slot > 0);
    }
  }
}

// The bounds of a page's tokens from slot `first` to n - 1, from their keys in
// the cache, by a workgroup; those there already count for the slots before.
template <typename T, int D>
__device__ __forceinline__ void bounds_of_page(const AppendArgs& a, int32_t page, int g, int32_t first, int32_t n,
                                               float (*red)[32]) {
  constexpr int C = D / 16, ES = int(sizeof(T)), LANES = 256 / C;
  const int c = threadIdx.x % C;
  char* row = a.bounds + (int64_t(page) * a.Hkv + g) * (2 * D * ES);
  OldBounds<T> old;
  if (int(threadIdx.x) < C && first > 0) old.load(row, D, c, c + C);
  Bounds16 bd;
  bd.clear();
  for (int32_t t = first + int32_t(threadIdx.x) / C; t < n; t += LANES) {
    const char* src = a.kp + slot_offset(a.ks, Slot{page, t, true}, g);
    float y[16];
    load8<T>(y, src + c * 8 * ES);
    load8<T>(y + 8, src + (c + C) * 8 * ES);
#pragma unroll
    for (int e = 0; e < 16; ++e) bd.add(e, y[e]);
  }
  join_bounds<C>(bd, red);
  if (int(threadIdx.x) < C) store_bounds<T, D>(bd, old, row, c, c + C, first > 0);
}
// Of every page of the sequences.
template <typename T, int D>
__global__ __launch_bounds__(256) void page_bounds(AppendArgs a) {
  __shared__ float red[4 * (D / 16)][32];
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv;
  const int32_t len = seq_len(a.lens, b, a.cap);
  for (int32_t i = blockIdx.y; (int64_t(i) << a.shift) < len; i += gridDim.y) {
    const int32_t page = a.table[int64_t(b) * a.max_pages + i];
    if (uint32_t(page) >= uint32_t(a.n_pages)) continue;
    const int32_t left = len - (i << a.shift);
    bounds_of_page<T, D>(a, page, g, 0, left < (1 << a.shift) ? left : 1 << a.shift, red);
    __syncthreads();
  }
}
// Of the pages that an append wrote to (a workgroup per page and KV head): the
// new keys joined to what is there, as append_rotated does it, so that which of
// the two keeps the bounds shows in none of them.
template <typename T, int D>
__global__ __launch_bounds__(256) void new_bounds(AppendArgs a, PagedSeqs s) {
  __shared__ float red[4 * (D / 16)][32];
  const int tile = int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  const int si = find_seq(s, tile), b = s.seq0 + si;
  const int32_t len = seq_len(a.lens, b, a.cap), p0 = len - s.len[si] > 0 ? len - s.len[si] : 0;
  const int32_t i = (p0 >> a.shift) + (tile - s.tile0[si]);
  if ((int64_t(i) << a.shift) >= len) return;
  const int32_t page = a.table[int64_t(b) * a.max_pages + i];
  if (uint32_t(page) >= uint32_t(a.n_pages)) return;
  const int32_t u0 = i << a.shift, left = len - u0;
  bounds_of_page<T, D>(a, page, g, p0 > u0 ? p0 - u0 : 0, left < (1 << a.shift) ? left : 1 << a.shift, red);
}

// The last tokens of every sequence as rows of the call's type: a thread has
// eight elements of a key and of a value.
template <typename T, int D>
__global__ __launch_bounds__(256) void read_rows4(AppendArgs a, PagedSeqs s, char* ko, char* vo) {
  constexpr int P = D / 8, ES = int(sizeof(T));
  const int tile = int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  const int si = find_seq(s, tile), b = s.seq0 + si, ntok = s.len[si];
  const int32_t len = seq_len(a.lens, b, a.cap), p0 = len - ntok;
  const int32_t i0 = (tile - s.tile0[si]) << a.unit, i1 = ntok - i0 < (1 << a.unit) ? ntok : i0 + (1 << a.unit);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int c = threadIdx.x % P;
  for (int32_t i = i0 + int32_t(threadIdx.x) / P; i < i1; i += 256 / P) {
    const int32_t j = p0 + i;
    Slot sl = {0, 0, false};
    if (j >= 0) sl = paged_slot(trow, j, a.shift, a.n_pages);
    const int64_t to = ((int64_t(s.start[si]) + i) * a.Hkv + g) * (D * ES) + c * 8 * ES;
    const int64_t at = ((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot;
#pragma unroll
    for (int kv = 0; kv < 2; ++kv) {
      uint4 w = make_uint4(0, 0, 0, 0);
      if (sl.ok) {
        const uint8_t* codes = (kv ? a.p4.vc : a.p4.kc) + at * (D / 2);
        const uint8_t* scales = (kv ? a.p4.vs : a.p4.ks) + at * (D / kGroup4);
        w = bf16_of_codes(*reinterpret_cast<const uint32_t*>(codes + 4 * c), scale_of(scales[c / 4]));
      }
      if constexpr (ES == 2) {
        *reinterpret_cast<uint4*>((kv ? vo : ko) + to) = w;
      } else {
        Frag<bf16_t> f;
        f.v = w;
        float y[8];
        f.to_floats(y);
        store8<T>((kv ? vo : ko) + to, y);
      }
    }
  }
}

template <typename T, int D, bool FOUR>
hipError_t append_t(const AppendArgs& a, const PagedSeqs& s, bool interleaved, hipStream_t stream) {
  const bool single = std::all_of(s.len, s.len + s.nseq, [](int32_t n) { return n == 1; });
  const uint32_t n = uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv);
  if (n == 0) return hipSuccess;
  if (single) {
    if (interleaved) append_rotated<T, D, FOUR, true, true><<<n, 256, 0, stream>>>(a, s);
    else append_rotated<T, D, FOUR, false, true><<<n, 256, 0, stream>>>(a, s);
  } else {
    if (interleaved) append_rotated<T, D, FOUR, true, false><<<n, 256, 0, stream>>>(a, s);
    else append_rotated<T, D, FOUR, false, false><<<n, 256, 0, stream>>>(a, s);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_append(const AppendArgs& a, const PagedSeqs& s, int d, int dtype, bool four, bool interleaved,
                         hipStream_t stream) {
  if (dtype == GLIDE_BF16) {
    if (d == 128)
      return four ? append_t<bf16_t, 128, true>(a, s, interleaved, stream)
                  : append_t<bf16_t, 128, false>(a, s, interleaved, stream);
    return four ? append_t<bf16_t, 64, true>(a, s, interleaved, stream)
                : append_t<bf16_t, 64, false>(a, s, interleaved, stream);
  }
  if (d == 128)
    return four ? append_t<float, 128, true>(a, s, interleaved, stream)
                : append_t<float, 128, false>(a, s, interleaved, stream);
  return four ? append_t<float, 64, true>(a, s, interleaved, stream)
              : append_t<float, 64, false>(a, s, interleaved, stream);
}

hipError_t launch_page_bounds(const AppendArgs& a, int64_t keys, int d, int dtype, hipStream_t stream) {
  const int64_t pages = (keys + (int64_t(1) << a.shift) - 1) >> a.shift;
  const dim3 grid(uint32_t(a.B * a.Hkv), uint32_t(std::max<int64_t>(1, std::min<int64_t>(pages, 4096))));
  if (dtype == GLIDE_BF16) {
    if (d == 128) page_bounds<bf16_t, 128><<<grid, 256, 0, stream>>>(a);
    else page_bounds<bf16_t, 64><<<grid, 256, 0, stream>>>(a);
  } else {
    if (d == 128) page_bounds<float, 128><<<grid, 256, 0, stream>>>(a);
    else page_bounds<float, 64><<<grid, 256, 0, stream>>>(a);
  }
  return hipGetLastError();
}

hipError_t launch_new_bounds(const AppendArgs& a, const PagedSeqs& s, int d, int dtype, hipStream_t stream) {
  const uint32_t n = uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv);
  if (n == 0) return hipSuccess;
  if (dtype == GLIDE_BF16) {
    if (d == 128) new_bounds<bf16_t, 128><<<n, 256, 0, stream>>>(a, s);
    else new_bounds<bf16_t, 64><<<n, 256, 0, stream>>>(a, s);
  } else {
    if (d == 128) new_bounds<float, 128><<<n, 256, 0, stream>>>(a, s);
    else new_bounds<float, 64><<<n, 256, 0, stream>>>(a, s);
  }
  return hipGetLastError();
}

hipError_t launch_read4(const AppendArgs& a, const PagedSeqs& s, char* ko, char* vo, int d, int dtype,
                        hipStream_t stream) {
  const uint32_t n = uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv);
  if (n == 0) return hipSuccess;
  if (dtype == GLIDE_BF16) {
    if (d == 128) read_rows4<bf16_t, 128><<<n, 256, 0, stream>>>(a, s, ko, vo);
    else read_rows4<bf16_t, 64><<<n, 256, 0, stream>>>(a, s, ko, vo);
  } else {
    if (d == 128) read_rows4<float, 128><<<n, 256, 0, stream>>>(a, s, ko, vo);
    else read_rows4<float, 64><<<n, 256, 0, stream>>>(a, s, ko, vo);
  }
  return hipGetLastError();
}

}  // namespace glide
