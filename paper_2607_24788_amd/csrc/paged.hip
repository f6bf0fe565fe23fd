// Softmax attention over a paged key-value cache: sliding window, sinks,
// grouped query heads, pieces of long rows joined, attention weights.
#include <algorithm>
#include <type_traits>

#include "paged.h"

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

// Orders a wave's own LDS accesses for the compiler (the hardware keeps them
// in order).
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ int32_t seq_len(const PagedArgs& a, int b) {
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : n > a.cap ? a.cap : n;
}

// ---------------------------------------------------------------------------
// NaN and infinities in value rows.  In a tile that some rows of a workgroup
// see and others do not (an "edge"), a weight of 0 must leave out what it
// multiplies, and 0 times infinity does not.  There such elements are staged as
// zeros, and the rows that do see them add their products one by one: work for
// nothing but such values.
__device__ __forceinline__ bool finite16(uint4 v, bf16_t) {
  auto two = [](uint32_t x) { return (x & 0x7f80u) != 0x7f80u && (x & 0x7f800000u) != 0x7f800000u; };
  return two(v.x) && two(v.y) && two(v.z) && two(v.w);
}
__device__ __forceinline__ bool finite16(uint4 v, float) {
  auto one = [](uint32_t x) { return (x & 0x7f800000u) != 0x7f800000u; };
  return one(v.x) && one(v.y) && one(v.z) && one(v.w);
}
__device__ __forceinline__ uint4 without_nonfinite(uint4 v, bf16_t) {
  auto two = [](uint32_t x) {
    return ((x & 0x7f80u) == 0x7f80u ? 0u : x & 0xffffu) | ((x & 0x7f800000u) == 0x7f800000u ? 0u : x & 0xffff0000u);
  };
  return make_uint4(two(v.x), two(v.y), two(v.z), two(v.w));
}
__device__ __forceinline__ uint4 without_nonfinite(uint4 v, float) {
  auto one = [](uint32_t x) { return (x & 0x7f800000u) == 0x7f800000u ? 0u : x; };
  return make_uint4(one(v.x), one(v.y), one(v.z), one(v.w));
}
// Four consecutive elements of a row, where not finite times w, added to y.
// (Nothing moves across: a batch of these loads would take the registers of
// the path that never comes here.)
__device__ __forceinline__ void add_nonfinite4(float* y, gptr_t p, float w, bf16_t) {
  const uint64_t x = *(const uint64_t __attribute__((address_space(1)))*)p;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t e = uint32_t(x >> (16 * i)) & 0xffffu;
    if ((e & 0x7f80u) == 0x7f80u) y[i] += w * to_f32(bf16_t(e));
  }
  __builtin_amdgcn_sched_barrier(0);
}
__device__ __forceinline__ void add_nonfinite4(float* y, gptr_t p, float w, float) {
  const uint4 x = gload16<false>(p);
  const uint32_t e[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if ((e[i] & 0x7f800000u) == 0x7f800000u) y[i] += w * __uint_as_float(e[i]);
  __builtin_amdgcn_sched_barrier(0);
}
// Bit r of the answer: some lane of r's LPR lanes, from lane r * LPR on, is set in m.
template <int LPR>
__device__ __forceinline__ uint32_t rows_of(uint64_t m) {
  uint32_t x = 0;
#pragma unroll
  for (int r = 0; r < 64 / LPR; ++r)
    x |= ((m >> (r * LPR)) & (LPR == 64 ? ~uint64_t(0) : (uint64_t(1) << (LPR & 63)) - 1)) ? 1u << r : 0u;
  return x;
}
// Whether the query at position t sees a cached token at position j.
__device__ __forceinline__ bool sees(const PagedArgs& a, int32_t j, int32_t t) {
  return (j <= t) & ((j > t - a.W) | (j < a.ns));
}
// Whether a tile of keys at positions j0 .. j1 holds any that one of the rows at
// t0 .. t1 does not see (and another may).
__device__ __forceinline__ bool edge_tile(const PagedArgs& a, int32_t j0, int32_t j1, int32_t t0, int32_t t1) {
  return j1 > t0 || (j0 <= t1 - a.W && j1 >= a.ns);
}

// ---------------------------------------------------------------------------
// A call's new rows of one KV head, tokens i0 <= i < i1 of a sequence, into
// their pages, by the workgroup whose row tile has their first head; the
// attention itself reads them where the call gave them.  Their weights start
// from 0.
template <int RB>  // bytes of a row
__device__ __forceinline__ void append_rows(const PagedArgs& a, const int32_t* trow, int g, int64_t tok0, int32_t p0,
                                            int32_t i0, int32_t i1) {
  constexpr int P = RB / 16;
  const int c = (threadIdx.x % P) * 16;
  for (int32_t i = i0 + int32_t(threadIdx.x / P); i < i1; i += 256 / P) {
    const int32_t j = p0 + i;
    if (j < 0) continue;
    const Slot sl = paged_slot(trow, j, a.shift, a.n_pages);
    if (!sl.ok) continue;
    const int64_t src = ((tok0 + i) * a.Hkv + g) * RB + c;
    const uint4 k = gload16<false>((gptr_t)a.kn + src), v = gload16<false>((gptr_t)a.vn + src);
    *reinterpret_cast<uint4*>(a.kp + slot_offset(a.ks, sl, g) + c) = k;
    *reinterpret_cast<uint4*>(a.vp + slot_offset(a.vs, sl, g) + c) = v;
    if (a.wp && c == 0) a.wp[((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot] = 0.f;
  }
}
// The tokens whose first head is in rows [r0, r0 + n) of a tile.
__device__ __forceinline__ int32_t first_token(int r0, int G) { return (r0 + G - 1) / G; }

// ---------------------------------------------------------------------------
// Attention of one tile of 16 rows ((token, head) pairs of one KV head) over
// one piece of the tokens that they see; the four waves take tiles of 32 keys
// in turn, each with a running maximum and sum of its own, joined at the end.
//   S^T = K Q^T (keys are the MFMA rows): a lane holds 8 scores of one row,
//   already the right operand of O^T += V^T P^T with keys in the order
//   4g + 0..3, 16 + 4g + 0..3; V goes through LDS for its columns.
// Decode is bound by HBM: 32 sequences of 16K..32K tokens, 8 KV heads of 128,
// bf16, 3.2 GB in 530 us (6.0 TB/s); 8 sequences of 16K in fp32 5.5 TB/s.
// Small calls are bound by the chain table -> rows -> scores -> join of the
// waves: 5.7 us over 64 tokens.
struct NoSeqs {};
template <typename T, int D, typename Seqs>  // Seqs: PagedSeqs, or NoSeqs for a decode call
__global__ __launch_bounds__(256, 2) void attend_rows(PagedArgs a, Seqs s) {
  constexpr bool DECODE = std::is_same<Seqs, NoSeqs>::value;
  constexpr int KK = D / 32, CT = D / 16, ES = int(sizeof(T));
  // LDS rows: 32 bytes longer in bf16 (eight consecutive K rows' pieces, and
  // four V rows' 32-byte segments, in different banks), 16 in fp32 (V alone)
  constexpr bool KLDS = ES == 2;
  constexpr int RS = D + (KLDS ? 16 : 4), LPR = D * ES / 16, RPI = 64 / LPR, NL = kPagedTile / RPI;
  __shared__ __align__(16) T klds[KLDS ? 4 : 1][KLDS ? kPagedTile * RS : 1];
  __shared__ __align__(16) T vlds[4][kPagedTile * RS];
  __shared__ float sm[4][16], sl_[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, lg = lane >> 4;
  int b, g, r0, nrow, p0, ntok;
  int64_t tok0;
  if constexpr (DECODE) {
    b = blockIdx.x / a.Hkv;
    g = blockIdx.x % a.Hkv;
    r0 = 0;
    ntok = 1;
    tok0 = b;
  } else {
    const int tile = blockIdx.x / a.Hkv, i = find_seq(s, tile);
    g = blockIdx.x % a.Hkv;
    b = s.seq0 + i;
    r0 = (tile - s.tile0[i]) * kPagedRows;
    ntok = s.len[i];
    tok0 = s.start[i];
  }
  nrow = ntok * a.G;
  const int unit = DECODE && a.per_head ? int(blockIdx.x) : b;
  const int32_t len = seq_len(a, unit);
  p0 = len - ntok;
  const int rl = nrow - 1 - r0 < kPagedRows - 1 ? nrow - 1 - r0 : kPagedRows - 1;  // last row of the tile
  const int32_t t0 = p0 + r0 / a.G > 0 ? p0 + r0 / a.G : 0, t1 = p0 + (r0 + rl) / a.G;
  // this lane's row
  const bool rok = n <= rl;
  const int r = r0 + (rok ? n : rl);
  const int32_t tr = rok ? p0 + r / a.G : -1;
  const int64_t orow = (tok0 + r / a.G) * a.Hq + g * a.G + r % a.G;  // row of q, out, lse
  Seen sn = {0, 0, 0};
  if (t1 >= 0) sn = seen_by(t0, t1, a.W, a.ns);
  int32_t pl = (sn.n + a.npiece - 1) / a.npiece;
  pl = pl > a.piece ? (pl + 127) & ~127 : a.piece;
  // (v0 in 64 bits: blockIdx.y * pl may pass 2^31 where pieces are longer than they need be)
  const int32_t v0 = int32_t(int64_t(blockIdx.y) * pl < sn.n ? int64_t(blockIdx.y) * pl : sn.n);
  const int32_t v1 = sn.n - v0 > pl ? v0 + pl : sn.n;
  const int32_t* trow = a.table + int64_t(unit) * a.max_pages;
  const gptr_t zr = (gptr_t)zero_row;

  Frag<T> qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    qf[kk].load(reinterpret_cast<const T*>(a.q) + orow * D + 32 * kk + 8 * lg);
    if (!rok) qf[kk].zero();
  }
  float m = kNoMax, l = 0.f;
  f32x4_t acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = zero4();
  T* vt = vlds[wave];

  if (a.kn && blockIdx.y == 0) {
    const int32_t end = first_token(r0 + kPagedRows, a.G);
    append_rows<D * ES>(a, trow, g, tok0, p0, first_token(r0, a.G), end < ntok ? end : ntok);
  }

  // Tiles are read one ahead: a tile's rows are asked for as soon as the one
  // before it is out of the registers, its page numbers a tile earlier.
  // bf16: whole rows by neighbouring lanes (16 bytes each), K and V through
  // LDS.  fp32: a K fragment's four lanes read whole lines; V alone goes
  // through LDS.
  constexpr int NR = KLDS ? 1 : 2;  // rows that a lane looks up: n + 16t, or lane % 32
  struct At {
    int32_t j[NR], page[NR];  // position (-1: behind the piece) and page
  };
  auto look = [&](int32_t x) {
    At p;
#pragma unroll
    for (int t = 0; t < NR; ++t) {
      const int32_t vi = x + (KLDS ? lane & 31 : 16 * t + n);
      p.j[t] = vi < v1 ? sn.pos(vi) : -1;
      p.page[t] = trow[(vi < v1 ? p.j[t] : 0) >> a.shift];
    }
    return p;
  };
  // a row's address: the cache's, the call's new row, or zeros
  auto row_at = [&](bool good, int32_t j, int32_t page, gptr_t* kr, gptr_t* vr) {
    const Slot sl = {page, j & ((1 << a.shift) - 1), true};
    *kr = good ? (gptr_t)a.kp + slot_offset(a.ks, sl, g) : zr;
    *vr = good ? (gptr_t)a.vp + slot_offset(a.vs, sl, g) : zr;
    if (a.kn && good && j >= p0) {
      const int64_t at = ((tok0 + j - p0) * a.Hkv + g) * (D * ES);
      *kr = (gptr_t)a.kn + at;
      *vr = (gptr_t)a.vn + at;
    }
  };
  // the values of key `key` of a tile (position j) that are not finite, for the rows that see it
  auto add_nonfinite = [&](int key, int32_t j, const float* p) {
    float w = -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) w = i == ((key >> 4) * 4 + (key & 3)) ? p[i] : w;
    w = __shfl(__builtin_amdgcn_exp2f(w - m), ((key >> 2) & 3) * 16 + n);
    gptr_t kr, vr;
    row_at(true, j, trow[j >> a.shift], &kr, &vr);
    if (!sees(a, j, tr)) return;  // (not by the weight, which may underflow)
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      float y[4] = {acc[ct][0], acc[ct][1], acc[ct][2], acc[ct][3]};
      add_nonfinite4(y, vr + (16 * ct + 4 * lg) * ES, w, T());
      acc[ct] = f32x4_t{y[0], y[1], y[2], y[3]};
    }
  };
  Frag<T> kf[2][KK], vf[2][KK];  // bf16: NL pieces each, [0] and [1] in turn
  uint32_t okm = 0;              // the tile's rows that are there
  auto fetch = [&](const At& p, int32_t x) {
    if constexpr (KLDS) {
      const bool good = p.j[0] >= 0 && uint32_t(p.page[0]) < uint32_t(a.n_pages);
      okm = uint32_t(__ballot(good));
      const int32_t page = good ? p.page[0] : -1;
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        const int row = e * RPI + lane / LPR;
        const int32_t pe = __shfl(page, row);
        gptr_t kr, vr;
        row_at(pe >= 0, sn.pos(x + row), pe, &kr, &vr);
        gload_frag<DECODE>(kf[e / KK][e % KK], kr + (lane % LPR) * 16);
        gload_frag<DECODE>(vf[e / KK][e % KK], vr + (lane % LPR) * 16);
      }
    } else {
      okm = 0;
#pragma unroll
      for (int t = 0; t < NR; ++t) {
        const bool good = p.j[t] >= 0 && uint32_t(p.page[t]) < uint32_t(a.n_pages);
        gptr_t kr, vr;
        row_at(good, p.j[t], p.page[t], &kr, &vr);
        okm |= (uint32_t(__ballot(good)) & 0xffffu) << (16 * t);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) gload_frag<DECODE>(kf[t][kk], kr + (32 * kk + 8 * lg) * ES);
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) gload_frag<DECODE>(vf[t][kk], vr + (32 * kk + 8 * lg) * ES);
      }
    }
  };
  // rows of the fetched tile with values that are not finite (lane: of its pieces)
  auto edge = [&](int32_t x) { return edge_tile(a, sn.pos(x), sn.pos(x + kPagedTile - 1), t0, t1); };
  auto nonfinite_rows = [&]() {
    uint32_t bad = 0;
    if constexpr (KLDS) {
#pragma unroll
      for (int e = 0; e < NL; ++e)
        bad |= rows_of<LPR>(__ballot(!finite16(vf[e / KK][e % KK].v, T()))) << (e * RPI);
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bool nf = false;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
          for (int e = 0; e < 8; ++e) nf |= (__float_as_uint(vf[t][kk].v[e]) & 0x7f800000u) == 0x7f800000u;
        const uint64_t m4 = __ballot(nf);
        bad |= uint32_t((m4 | m4 >> 16 | m4 >> 32 | m4 >> 48) & 0xffffu) << (16 * t);
      }
    }
    return bad;
  };
  auto drop_nonfinite = [&]() {
    const bool any = nonfinite_rows() != 0;
    if (any) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          if constexpr (KLDS) {
            vf[t][kk].v = without_nonfinite(vf[t][kk].v, T());
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              vf[t][kk].v[e] = (__float_as_uint(vf[t][kk].v[e]) & 0x7f800000u) == 0x7f800000u ? 0.f : vf[t][kk].v[e];
          }
        }
    }
    return any;
  };
  // scores of the lane's keys 16 t + 4 lg + i in p[4 t + i], -inf where its row does not see them
  auto masked = [&](const f32x4_t* sc, uint32_t okc, int32_t x, float* p) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 4 * lg + i;
        bool see = (okc >> (16 * t + key)) & 1;
        if constexpr (!DECODE) {
          const int32_t j = sn.pos(x + 16 * t + key);
          see = see && j <= tr && (j > tr - a.W || j < a.ns);
        }
        p[4 * t + i] = see ? sc[t][i] * a.scale : -INFINITY;
      }
  };
  bool any_bad = false;
  constexpr int STEP = 4 * kPagedTile;
  int32_t x = v0 + wave * kPagedTile;
  At next = {};
  if (x < v1) {
    const At first = look(x);
    next = look(x + STEP);
    fetch(first, x);
  }
  for (; x < v1; x += STEP) {
    f32x4_t sc[2] = {zero4(), zero4()};
    const uint32_t okc = okm;
    if constexpr (!DECODE) {
      if (edge(x)) any_bad |= drop_nonfinite();
    }
    if constexpr (KLDS) {
      T* kt = klds[wave];
#pragma unroll
      for (int e = 0; e < NL; ++e) {
        const int at = (e * RPI + lane / LPR) * RS + (lane % LPR) * 8;
        *reinterpret_cast<uint4*>(kt + at) = kf[e / KK][e % KK].v;
        *reinterpret_cast<uint4*>(vt + at) = vf[e / KK][e % KK].v;
      }
      wave_lds_order();
      if (x + STEP < v1) {
        const At now = next;
        next = look(x + 2 * STEP);
        fetch(now, x + STEP);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          Frag<T> k;
          k.load(kt + (16 * t + n) * RS + 32 * kk + 8 * lg);
          sc[t] = mma(k, qf[kk], sc[t]);
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
      if (x + STEP < v1) {
        const At now = next;
        next = look(x + 2 * STEP);
        fetch(now, x + STEP);
      }
    }
    float p[8];
    masked(sc, okc, x, p);
    float mx = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, p[i]);
    if constexpr (DECODE) {
      if (a.scores && rok) {
        float* w = a.scores + (int64_t(b) * a.Hq + g * a.G + r) * a.nv + x + 4 * lg;
#pragma unroll
        for (int t = 0; t < 2; ++t)
          *reinterpret_cast<float4*>(w + 16 * t) = make_float4(p[4 * t], p[4 * t + 1], p[4 * t + 2], p[4 * t + 3]);
      }
    }
    mx = lg_max(mx);
    const float f = __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    l *= f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      p[i] = __builtin_amdgcn_exp2f(p[i] - m);
      l += p[i];
    }
    Frag<T> pf;
    pf.set8(p);  // bf16: weights rounded to half a step, 2^-8 of each at most
    wave_lds_order();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[ct][i] *= f;
      Frag<T> vc;
      load_colfrag2(vc, vt, RS, 4 * lg, 16 + 4 * lg, 16 * ct);
      acc[ct] = mma(vc, pf, acc[ct]);
    }
    wave_lds_order();
  }
  if constexpr (!DECODE) {
    // Nearly never: the edges that were staged without some of their values.
    if (any_bad) {
#pragma unroll 1
      for (x = v0 + wave * kPagedTile; x < v1; x += STEP) {
        if (!edge(x)) continue;
        fetch(look(x), x);
        uint32_t bad = nonfinite_rows();
        f32x4_t sc[2] = {zero4(), zero4()};
        if constexpr (KLDS) {
          T* kt = klds[wave];
#pragma unroll
          for (int e = 0; e < NL; ++e)
            *reinterpret_cast<uint4*>(kt + (e * RPI + lane / LPR) * RS + (lane % LPR) * 8) = kf[e / KK][e % KK].v;
          wave_lds_order();
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int kk = 0; kk < KK; ++kk) {
            Frag<T> k = kf[t][kk];
            if constexpr (KLDS) k.load(klds[wave] + (16 * t + n) * RS + 32 * kk + 8 * lg);
            sc[t] = mma(k, qf[kk], sc[t]);
          }
        wave_lds_order();
        float p[8];
        masked(sc, okm, x, p);
        while (bad) {
          const int key = __builtin_ctz(bad);
          bad &= bad - 1;
          add_nonfinite(key, sn.pos(x + key), p);
        }
      }
    }
  }

  // the four waves' parts: each row's frame, then the sums in it
  l = lg_sum(l);
  if (lane < 16) {
    sm[wave][lane] = m;
    sl_[wave][lane] = l;
  }
  __syncthreads();
  float M = kNoMax, L = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w][n]);
#pragma unroll
  for (int w = 0; w < 4; ++w) L += sl_[w][n] * __builtin_amdgcn_exp2f(sm[w][n] - M);
  const float f = __builtin_amdgcn_exp2f(m - M);
  // acc through LDS, one wave after the other's in a fixed order: [row][d] fp32
  float* red = reinterpret_cast<float*>(&vlds[0][0]);
  constexpr int RD = D + 4;
  for (int w = 0; w < 4; ++w) {
    if (wave == w) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float* at = red + n * RD + 16 * ct + 4 * lg + i;
          const float y = acc[ct][i] * f;
          *at = w == 0 ? y : *at + y;
        }
    }
    __syncthreads();
  }
  const bool split = a.npiece > 1 || (DECODE && a.scores);  // join_weights joins one piece too
  if (wave == 0 && lane < 16 && rok) {
    if (split) {
      float* ml = a.ml + (orow * a.npiece + blockIdx.y) * 2;
      ml[0] = M;
      ml[1] = L;
    } else {
      const float lse2 = L > 0.f ? M + __builtin_amdgcn_logf(L) : L == 0.f ? -INFINITY : L;
      if (a.lse) a.lse[orow] = lse2 * kLn2;
      if (a.lse2) a.lse2[orow] = lse2;
    }
  }
  // 16 threads per row, D / 16 consecutive elements each
  const int rr = threadIdx.x >> 4, e0 = (threadIdx.x & 15) * (D / 16);
  if (rr > rl) return;
  float Lr = 0.f, Mr = kNoMax;
#pragma unroll
  for (int w = 0; w < 4; ++w) Mr = fmaxf(Mr, sm[w][rr]);
#pragma unroll
  for (int w = 0; w < 4; ++w) Lr += sl_[w][rr] * __builtin_amdgcn_exp2f(sm[w][rr] - Mr);
  const int r2 = r0 + rr;
  const int64_t o2 = (tok0 + r2 / a.G) * a.Hq + g * a.G + r2 % a.G;
  if (split) {
    float* w = a.acc + (o2 * a.npiece + blockIdx.y) * D + e0;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) w[e] = red[rr * RD + e0 + e];
  } else {
    const float inv = Lr == 0.f ? 0.f : 1.f / Lr;
    T* w = reinterpret_cast<T*>(a.out) + o2 * D + e0;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) w[e] = from_f32<T>(red[rr * RD + e0 + e] * inv);
  }
}

// ---------------------------------------------------------------------------
// Attention of many rows (bf16): a workgroup takes 128 rows ((token, head)
// pairs of one KV head, 32 per wave) over the 64-key tiles that any of them
// sees, K and V staged in LDS for the four waves.
//   S^T = K Q^T with 32x32x16 MFMAs: a lane holds the scores of one row, 16 of
//   each 32 keys, in the order that the right operand of O^T += V^T P^T takes
//   (keys 8j + 4h + 0..3 of lane half h), so the weights never leave its
//   registers; V^T comes from the transposing LDS reads.
//   Row sums of the weights are taken before they are rounded to bf16: lse is
//   exact to fp32.  The frame (a row's maximum) moves only when a score passes
//   it by 2^8: weights up to 2^8 round alike, and fp32 sums hold them.
// Bound by the matrix cores at the clock that the power limit leaves: a prompt
// of 32768 tokens (32 / 8 heads of 128) 9.1 ms = 969 TFLOP/s, MFMAs half of
// the cycles at 1.94 GHz; 8192 tokens with W = 2048 301 us.  Tiles are staged
// through registers, a tile ahead: two workgroups per CU (64 KB of LDS, 241
// registers each).
// A 16-byte piece c of row r is kept at piece c ^ swz(r) of the row: eight
// consecutive rows' K pieces, and four rows' 64-byte V segments, lie in
// different banks.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
typedef float f32x16_t __attribute__((ext_vector_type(16)));
__device__ __forceinline__ f32x16_t mma32(uint4 a, uint4 b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                 0, 0, 0);
}
__device__ __forceinline__ uint4 vt_frag(const char* p, const char* q) {
  const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(__attribute__((address_space(3))) char*)p);
  const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(__attribute__((address_space(3))) char*)q);
  const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
  return make_uint4(x.x, x.y, y.x, y.y);
}
// The block table through the scalar cache (nothing writes it during a call).
__device__ __forceinline__ int32_t table_at(const int32_t* row, int32_t i) {
  typedef const int32_t __attribute__((address_space(4))) * cptr;
  return ((cptr)(uintptr_t)row)[i];
}

// At a scalar offset more (which the check against the size counts too).
__device__ __forceinline__ uint4 bload16_at(brsrc_t r, uint32_t off, int32_t at) {
  return __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(r, off, at, 0));
}

template <int D>
__global__ __launch_bounds__(256, 2) void attend_tiles(PagedArgs a, PagedSeqs s) {
  constexpr int KK = D / 16, CT = D / 32, RB = 2 * D, LPR = RB / 16, RPI = 64 / LPR, NI = 16 / RPI;
  constexpr int KB = kTileKeys * RB;  // bytes of a K (or V) tile
  __shared__ __align__(16) char lds[2][2 * KB];
  // edges with values that are not finite: whether there are any; those of a
  // tile, by the 16 rows of a wave
  __shared__ uint32_t any_bad, bad[4];
  const int lane = threadIdx.x & 63, h = lane >> 5, q = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = s.tile0[s.nseq] - 1 - int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  const int si = find_seq(s, tile), b = s.seq0 + si, ntok = s.len[si];
  const int32_t len = __builtin_amdgcn_readfirstlane(seq_len(a, b)), p0 = len - ntok;
  const int r0 = (tile - s.tile0[si]) * kTileRows, rend = ntok * a.G;
  const int rlast = r0 + kTileRows < rend ? r0 + kTileRows - 1 : rend - 1;
  const int32_t t0 = p0 + r0 / a.G > 0 ? p0 + r0 / a.G : 0, t1 = p0 + rlast / a.G;
  // this wave's rows, and this lane's
  const int w0 = r0 + 32 * wave;
  const bool rok = w0 + q < rend;
  const int r = rok ? w0 + q : rend - 1, tok = r / a.G;
  const int32_t tr = rok ? p0 + tok : -1;
  const int64_t orow = (int64_t(s.start[si]) + tok) * a.Hq + g * a.G + (r - tok * a.G);
  const int32_t tw0 = p0 + (w0 < rend ? w0 : rend - 1) / a.G;
  const int32_t tw1 = w0 < rend ? p0 + (w0 + 31 < rend ? w0 + 31 : rend - 1) / a.G : -1;
  // tiles: those of the sinks before the window's, then the window's
  const int32_t wstart = t0 - a.W + 1 > 0 ? t0 - a.W + 1 : 0;
  int32_t nt = 0, nsink = 0, wt0 = 0;
  if (t1 >= 0) {
    wt0 = wstart / kTileKeys;
    nsink = (a.ns + kTileKeys - 1) / kTileKeys;
    nsink = nsink < wt0 ? nsink : wt0;
    nt = nsink + (t1 / kTileKeys >= wt0 ? t1 / kTileKeys - wt0 + 1 : 0);
  }
  int32_t per = (nt + a.npiece - 1) / a.npiece;
  per = per > a.piece / kTileKeys ? per : a.piece / kTileKeys;
  const int32_t i0 = int32_t(int64_t(blockIdx.y) * per < nt ? int64_t(blockIdx.y) * per : nt);
  const int32_t i1 = nt - i0 > per ? i0 + per : nt;
  auto key0 = [&](int32_t i) { return (i < nsink ? i : wt0 + i - nsink) * kTileKeys; };
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int32_t last_entry = (t1 > 0 ? t1 : 0) >> a.shift;

  uint4 qf[KK];
  {
    const char* qp = a.q + orow * RB + 16 * h;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      qf[kk] = *reinterpret_cast<const uint4*>(qp + 32 * kk);
      if (!rok) qf[kk] = make_uint4(0, 0, 0, 0);
    }
    if (a.scale < 0) {  // scores of -q: the frame is a maximum of raw scores
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        qf[kk].x ^= 0x80008000u;
        qf[kk].y ^= 0x80008000u;
        qf[kk].z ^= 0x80008000u;
        qf[kk].w ^= 0x80008000u;
      }
    }
  }
  const float c = fabsf(a.scale);

  // staging: row 16 wave + RPI i + lane / LPR of a tile, piece lane % LPR
  const int srow = lane / LPR;
  uint32_t koff[NI], voff[NI], noff[NI];  // in the pools, and among the call's new rows
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int rr = RPI * i + srow, piece = (lane % LPR) ^ swz<D>(rr);
    koff[i] = uint32_t(rr) * uint32_t(a.ks[2]) + piece * 16;
    voff[i] = uint32_t(rr) * uint32_t(a.vs[2]) + piece * 16;
    noff[i] = uint32_t(rr) * uint32_t(a.Hkv * RB) + piece * 16;
  }
  struct Stage {
    uint4 k[NI], v[NI];
  };
  // pages of a tile's four groups of 16 keys
  struct Pages {
    int32_t p[4];
  };
  auto pages_of = [&](int32_t i) {
    Pages x;
    const int32_t k0 = key0(i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int32_t at = (k0 + 16 * e) >> a.shift;
      x.p[e] = table_at(trow, at < last_entry ? at : last_entry);
    }
    return x;
  };
  // this sequence's new rows of the head, where the call gave them
  const int64_t nat = (int64_t(s.start[si]) * a.Hkv + g) * RB;
  const brsrc_t nkr = make_rsrc(a.kn + nat, kOOB), nvr = make_rsrc(a.vn + nat, kOOB);
  const int32_t new0 = a.kn ? p0 : 0x7fffffff;  // their first position
  auto fetch = [&](int32_t i, const Pages& pg, Stage& st) {
    const int32_t k0 = key0(i) + 16 * wave;
    const int32_t page = wave == 0 ? pg.p[0] : wave == 1 ? pg.p[1] : wave == 2 ? pg.p[2] : pg.p[3];
    const bool ok = uint32_t(page) < uint32_t(a.n_pages);
    // rows that some query of the workgroup sees: [lo, hi) of the 16, and those before sk
    const int32_t lo = wstart - k0, hi = t1 + 1 - k0, sk = (a.ns < t1 + 1 ? a.ns : t1 + 1) - k0;
    const bool whole = ok && ((lo <= 0 && hi >= 16) || sk >= 16);
    if (whole && k0 >= new0) {
      const int32_t at = (k0 - p0) * a.Hkv * RB;
#pragma unroll
      for (int e = 0; e < NI; ++e) {
        st.k[e] = bload16_at(nkr, noff[e], at);
        st.v[e] = bload16_at(nvr, noff[e], at);
      }
      return;
    }
    const int64_t slot = k0 & ((1 << a.shift) - 1), pp = ok ? page : 0;
    const brsrc_t kr = make_rsrc(a.kp + pp * a.ks[0] + g * a.ks[1] + slot * a.ks[2], kOOB);
    const brsrc_t vr = make_rsrc(a.vp + pp * a.vs[0] + g * a.vs[1] + slot * a.vs[2], kOOB);
    if (whole && new0 - k0 >= 16) {
#pragma unroll
      for (int e = 0; e < NI; ++e) {
        st.k[e] = bload16(kr, koff[e]);
        st.v[e] = bload16(vr, voff[e]);
      }
      return;
    }
    // row by row: from the pools, or among the new, or (not seen by any) zeros
#pragma unroll
    for (int e = 0; e < NI; ++e) {
      const int32_t rr = RPI * e + srow;
      const bool see = ok & (((rr >= lo) & (rr < hi)) | (rr < sk)), fresh = k0 + rr >= new0;
      const uint32_t off = (see & fresh) ? noff[e] + uint32_t(k0 - p0) * uint32_t(a.Hkv * RB) : kOOB;
      const uint4 x = bload16(nkr, off), y = bload16(nvr, off);
      const uint4 u = bload16(kr, (see & !fresh) ? koff[e] : kOOB), w = bload16(vr, (see & !fresh) ? voff[e] : kOOB);
      st.k[e] = make_uint4(u.x | x.x, u.y | x.y, u.z | x.z, u.w | x.w);
      st.v[e] = make_uint4(w.x | y.x, w.y | y.y, w.z | y.z, w.w | y.w);
    }
  };
  auto edge = [&](int32_t i) { return edge_tile(a, key0(i), key0(i) + kTileKeys - 1, t0, t1); };
  auto put = [&](int at, int32_t i, Stage& st) {
    char* w = lds[at] + wave * 16 * RB + lane * 16;
    if (edge(i)) {
#pragma unroll
      for (int e = 0; e < NI; ++e)
        if (__any(!finite16(st.v[e], bf16_t()))) {
          st.v[e] = without_nonfinite(st.v[e], bf16_t());
          any_bad = 1;
        }
    }
#pragma unroll
    for (int e = 0; e < NI; ++e) {
      *reinterpret_cast<uint4*>(w + e * 1024) = st.k[e];
      *reinterpret_cast<uint4*>(w + KB + e * 1024) = st.v[e];
    }
  };

  float mc = kNoMax, l = 0.f;
  f32x16_t o[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[ct][i] = 0.f;

  // per-lane LDS offsets: K row q of a 32-key half; V row i/4 (+ 4h) of a 16-key slab
  const int klane = q * RB, ksw = h ^ swz<D>(q);
  const int l16 = lane & 15, vrow = 4 * h + (l16 >> 2);
  const int vlane = KB + vrow * RB + (l16 & 1) * 8;
  const int vsw = (2 * ((lane >> 4) & 1) + ((l16 & 3) >> 1)) ^ swz<D>(vrow);

  auto key_of = [](int t, int e) { return 32 * t + 8 * (e >> 2) + (e & 3); };
  auto nothing = [&](int32_t k0) {  // for this wave in a tile
    return k0 > tw1 || (k0 + kTileKeys <= tw0 - a.W + 1 && k0 >= a.ns);
  };
  auto products = [&](const char* buf, f32x16_t* sc) {
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[t][e] = 0.f;
    }
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint4 kf = *reinterpret_cast<const uint4*>(buf + klane + 32 * t * RB + (((2 * kk) ^ ksw) << 4));
        sc[t] = mma32(kf, qf[kk], sc[t]);
      }
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int u = 0; u < KK - 3; ++u) {
      __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
    __builtin_amdgcn_s_setprio(0);
  };
  auto masks = [&](int32_t k0, uint32_t okp, f32x16_t* sc) {
    // what the rows do not see, where the tile may hold any (each kind tested
    // for the wave; key 32t + 8(e/4) + e%4 of the lane's is an instruction's
    // constant): keys after a row, keys before its window that are no sinks,
    // groups of 16 whose page is not there
    if (k0 + kTileKeys - 1 > tw0) {
      const int32_t last = tr - k0 - 4 * h;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[t][e] = key_of(t, e) > last ? -INFINITY : sc[t][e];
    }
    if (k0 <= tw1 - a.W && k0 + kTileKeys > a.ns) {
      const int32_t before = tr - a.W - k0 - 4 * h, sinks = a.ns - k0 - 4 * h;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          sc[t][e] = (key_of(t, e) <= before && key_of(t, e) >= sinks) ? -INFINITY : sc[t][e];
    }
    if (okp != 15u) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[t][e] = (okp >> (2 * t + (e >> 3))) & 1 ? sc[t][e] : -INFINITY;
    }
  };
  auto compute = [&](int at, int32_t i, uint32_t okp) {
    const char* buf = lds[at];
    const int32_t k0 = key0(i);
    if (nothing(k0)) return;
    f32x16_t sc[2];
    products(buf, sc);
    auto vfrag = [&](int sl, int ct) {
      const char* p = buf + vlane + 16 * sl * RB + (((4 * ct) ^ vsw) << 4);
      const char* p2 = buf + vlane + (16 * sl + 8) * RB + (((4 * ct) ^ vsw ^ 2) << 4);
      return vt_frag(p, p2);
    };
    uint4 vf[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) vf[ct] = vfrag(0, ct);
    masks(k0, okp, sc);
    float mx = sc[0][0];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, sc[t][e]);
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1])) * c;
    if (__any(mx > mc + 8.f)) {
      const float m2 = fmaxf(mc, mx), f = __builtin_amdgcn_exp2f(mc - m2);
      mc = m2;
      l *= f;
#pragma unroll
      for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[ct][e] *= f;
    }
    // P V by 16-key slabs: under a slab's MFMAs the next slab's weights are
    // taken and its V fragments read, in an order that the compiler keeps
    auto weights2 = [&](int sl, int e) {  // elements e, e + 1 of slab sl, as a bf16 pair
      float x = sc[sl >> 1][8 * (sl & 1) + e], y = sc[sl >> 1][8 * (sl & 1) + e + 1];
      x = __builtin_amdgcn_exp2f(fmaf(x, c, -mc));
      y = __builtin_amdgcn_exp2f(fmaf(y, c, -mc));
      l += x;
      l += y;
      return pack_bf16x2(x, y);
    };
    uint32_t pw[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) pw[e] = weights2(0, 2 * e);
    uint4 pf = make_uint4(pw[0], pw[1], pw[2], pw[3]);
#pragma unroll
    for (int sl = 0; sl < 4; ++sl) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        __builtin_amdgcn_sched_barrier(0);
        o[ct] = mma32(vf[ct], pf, o[ct]);
        if (sl < 3) {
          vf[ct] = vfrag(sl + 1, ct);
#pragma unroll
          for (int e = 0; e < 4 / CT; ++e) pw[ct * (4 / CT) + e] = weights2(sl + 1, 2 * (ct * (4 / CT) + e));
        }
      }
      pf = make_uint4(pw[0], pw[1], pw[2], pw[3]);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  if (a.kn && blockIdx.y == 0) {
    const int32_t end = first_token(r0 + kTileRows, a.G);
    append_rows<RB>(a, trow, g, s.start[si], p0, first_token(r0, a.G), end < ntok ? end : ntok);
  }

  if (threadIdx.x == 0) any_bad = 0;
  __syncthreads();
  if (i0 < i1) {
    auto okbits = [&](const Pages& p) {
      uint32_t m = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) m |= (uint32_t(p.p[e]) < uint32_t(a.n_pages) ? 1u : 0u) << e;
      return m;
    };
    Stage st;
    Pages pg = pages_of(i0);
    uint32_t okc = okbits(pg);
    fetch(i0, pg, st);
    pg = pages_of(i0 + 1 < i1 ? i0 + 1 : i0);
    put(0, i0, st);
    for (int32_t i = i0;; ++i) {
      const int cur = (i - i0) & 1;
      __syncthreads();
      const uint32_t okn = okbits(pg);
      if (i + 1 < i1) {
        fetch(i + 1, pg, st);
        pg = pages_of(i + 2 < i1 ? i + 2 : i + 1);
      }
      compute(cur, i, okc);
      if (i + 1 >= i1) break;
      put(cur ^ 1, i + 1, st);
      okc = okn;
    }
    __syncthreads();
    // Nearly never: the edges that were staged without some of their values,
    // once more, for the products that those values have.
    if (any_bad) {
#pragma unroll 1
      for (int32_t i = i0; i < i1; ++i) {
        if (!edge(i)) continue;
        pg = pages_of(i);
        fetch(i, pg, st);
        uint32_t rows = 0;
#pragma unroll
        for (int e = 0; e < NI; ++e) rows |= rows_of<LPR>(__ballot(!finite16(st.v[e], bf16_t()))) << (e * RPI);
        __syncthreads();
        if (lane == 0) bad[wave] = rows;
        put(0, i, st);
        __syncthreads();
        const int32_t k0 = key0(i);
        if (nothing(k0)) continue;
        f32x16_t sc[2];
        products(lds[0], sc);
        masks(k0, okbits(pg), sc);
#pragma unroll 1
        for (int u = 0; u < 4; ++u) {
          uint32_t m = __builtin_amdgcn_readfirstlane(bad[u]);
          while (m) {
            const int key = 16 * u + __builtin_ctz(m);
            m &= m - 1;
            // the key's weight: in lane half (key / 4) % 2, element 4 (key % 32 / 8) + key % 4 of half tile key / 32
            float x = -INFINITY;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int e = 0; e < 16; ++e) x = (key & ~4) == key_of(t, e) ? sc[t][e] : x;
            x = __builtin_amdgcn_exp2f(fmaf(x, c, -mc));
            const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
            x = __uint_as_float((key >> 2) & 1 ? both[1] : both[0]);
            const int32_t j = k0 + key;
            const Slot sl = paged_slot(trow, j, a.shift, a.n_pages);
            const gptr_t vr = j >= new0 ? (gptr_t)a.vn + nat + int64_t(j - p0) * a.Hkv * RB
                                        : (gptr_t)a.vp + slot_offset(a.vs, sl, g);
            if (!sees(a, j, tr)) continue;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                float y[4] = {o[ct][4 * e], o[ct][4 * e + 1], o[ct][4 * e + 2], o[ct][4 * e + 3]};
                add_nonfinite4(y, vr + (32 * ct + 8 * e + 4 * h) * 2, x, bf16_t());
#pragma unroll
                for (int w = 0; w < 4; ++w) o[ct][4 * e + w] = y[w];
              }
          }
        }
      }
    }
  }

  const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  if (a.npiece > 1) {
    if (!rok) return;
    const int64_t rec = orow * a.npiece + blockIdx.y;
    if (h == 0) {
      a.ml[rec * 2] = mc;
      a.ml[rec * 2 + 1] = l;
    }
    float* w = a.acc + rec * D + 4 * h;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<float4*>(w + 32 * ct + 8 * e) =
            make_float4(o[ct][4 * e], o[ct][4 * e + 1], o[ct][4 * e + 2], o[ct][4 * e + 3]);
    return;
  }
  if (rok && h == 0) {
    const float lse2 = l > 0.f ? mc + __builtin_amdgcn_logf(l) : l == 0.f ? -INFINITY : l;
    if (a.lse) a.lse[orow] = lse2 * kLn2;
    if (a.lse2) a.lse2[orow] = lse2;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  char* w = a.out + orow * RB + 16 * h;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int e = 0; e < 4; e += 2) {
      // elements 8e + 4h + 0..3 and 8(e+1) + 4h + 0..3 of the lane halves to 8e + 8h + 0..7
      uint32_t x[2][2];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        x[0][u] = pack_bf16x2(o[ct][4 * e + 2 * u] * inv, o[ct][4 * e + 2 * u + 1] * inv);
        x[1][u] = pack_bf16x2(o[ct][4 * e + 4 + 2 * u] * inv, o[ct][4 * e + 5 + 2 * u] * inv);
      }
      const auto y0 = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
      const auto y1 = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
      if (rok) *reinterpret_cast<uint4*>(w + 64 * ct + 16 * e) = make_uint4(y0[0], y1[0], y0[1], y1[1]);
    }
}

// ---------------------------------------------------------------------------
// Attention of many rows in fp32 (and in bf16 over pages of fewer than 16
// tokens): a workgroup takes 64 rows, 16 per wave, over the 32-key tiles that
// any of them sees, in turn; K and V go through LDS for the four waves, a tile
// ahead.  The products are those of attend_rows.  Bound by the fp32 matrix
// instructions (128 of 32 cycles per wave and tile at d = 128) and the address
// arithmetic between them: 4096 tokens, 32 / 8 heads of 128, 1.44 ms = 95
// TFLOP/s (attend_rows: 2.02 ms); bf16 over pages of 8, the same call 335 us =
// 411 TFLOP/s.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void attend_shared(PagedArgs a, PagedSeqs s) {
  constexpr int KK = D / 32, CT = D / 16, ES = int(sizeof(T)), RS = D + (ES == 2 ? 16 : 4);
  constexpr int LPR = D * ES / 16, RPI = 256 / LPR, NL = kPagedTile / RPI;  // rows of a load of the workgroup, loads
  static_assert(NL >= 1, "a tile holds a load's rows");
  __shared__ __align__(16) T kl[2][kPagedTile * RS], vl[2][kPagedTile * RS];
  __shared__ uint32_t any_bad, bad[4];  // as in attend_tiles; by the wave that read them
  const int lane = threadIdx.x & 63, n = lane & 15, lg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = s.tile0[s.nseq] - 1 - int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  const int si = find_seq(s, tile), b = s.seq0 + si, ntok = s.len[si];
  const int64_t tok0 = s.start[si];
  const int32_t len = __builtin_amdgcn_readfirstlane(seq_len(a, b)), p0 = len - ntok;
  const int r0 = (tile - s.tile0[si]) * kSharedRows, rend = ntok * a.G;
  const int rlast = r0 + kSharedRows < rend ? r0 + kSharedRows - 1 : rend - 1;
  const int32_t t0 = p0 + r0 / a.G > 0 ? p0 + r0 / a.G : 0, t1 = p0 + rlast / a.G;
  const int w0 = r0 + 16 * wave;
  const bool rok = w0 + n < rend;
  const int r = rok ? w0 + n : rend - 1, tok = r / a.G;
  const int32_t tr = rok ? p0 + tok : -1;
  const int64_t orow = (tok0 + tok) * a.Hq + g * a.G + (r - tok * a.G);
  const int32_t tw1 = w0 < rend ? p0 + (w0 + 15 < rend ? w0 + 15 : rend - 1) / a.G : -1;  // the wave's last position
  Seen sn = {0, 0, 0};
  if (t1 >= 0) sn = seen_by(t0, t1, a.W, a.ns);
  int32_t pl = (sn.n + a.npiece - 1) / a.npiece;
  pl = pl > a.piece ? (pl + 31) & ~31 : a.piece;
  const int32_t v0 = int32_t(int64_t(blockIdx.y) * pl < sn.n ? int64_t(blockIdx.y) * pl : sn.n);
  const int32_t v1 = sn.n - v0 > pl ? v0 + pl : sn.n;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;

  Frag<T> qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    qf[kk].load(reinterpret_cast<const T*>(a.q) + orow * D + 32 * kk + 8 * lg);
    if (!rok) qf[kk].zero();
  }
  float m = kNoMax, l = 0.f;
  f32x4_t acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = zero4();

  // rows RPI e + thread / LPR of a tile, 16 bytes of each: pages, then K and V
  const int srow = threadIdx.x / LPR, c16 = (threadIdx.x % LPR) * 16;
  struct Pages {
    int32_t p[NL];
  };
  auto look = [&](int32_t x) {
    Pages pg;
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int32_t vi = x + RPI * e + srow;
      pg.p[e] = trow[(vi < v1 ? sn.pos(vi) : 0) >> a.shift];
      if (vi >= v1) pg.p[e] = -1;
    }
    return pg;
  };
  const bool same = a.ks[0] == a.vs[0] && a.ks[1] == a.vs[1] && a.ks[2] == a.vs[2];
  uint4 ks[NL], vs[NL];
  auto fetch = [&](int32_t x, const Pages& pg) {
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int32_t j = sn.pos(x + RPI * e + srow);
      const bool ok = uint32_t(pg.p[e]) < uint32_t(a.n_pages);
      const Slot sl = {pg.p[e], j & ((1 << a.shift) - 1), true};
      const int64_t ko = slot_offset(a.ks, sl, g);
      int64_t vo = ko;
      if (!same) vo = slot_offset(a.vs, sl, g);
      gptr_t kr = ok ? (gptr_t)a.kp + ko : (gptr_t)zero_row;
      gptr_t vr = ok ? (gptr_t)a.vp + vo : (gptr_t)zero_row;
      if (a.kn && ok && j >= p0) {
        const int64_t at = ((tok0 + j - p0) * a.Hkv + g) * (D * ES);
        kr = (gptr_t)a.kn + at;
        vr = (gptr_t)a.vn + at;
      }
      ks[e] = gload16<false>(kr + c16);
      vs[e] = gload16<false>(vr + c16);
    }
  };
  // the tile's rows that are there, by row
  auto there = [&](int32_t x) {
    const int32_t vi = x + (lane & 31);
    const int32_t page = trow[(vi < v1 ? sn.pos(vi) : 0) >> a.shift];
    return uint32_t(__ballot(vi < v1 && uint32_t(page) < uint32_t(a.n_pages)));
  };
  auto edge = [&](int32_t x) { return edge_tile(a, sn.pos(x), sn.pos(x + kPagedTile - 1), t0, t1); };
  auto put = [&](int buf, int32_t x) {
    if (edge(x)) {
#pragma unroll
      for (int e = 0; e < NL; ++e)
        if (__any(!finite16(vs[e], T()))) {
          vs[e] = without_nonfinite(vs[e], T());
          any_bad = 1;
        }
    }
#pragma unroll
    for (int e = 0; e < NL; ++e) {
      const int at = (RPI * e + srow) * RS * ES + c16;
      *reinterpret_cast<uint4*>(reinterpret_cast<char*>(kl[buf]) + at) = ks[e];
      *reinterpret_cast<uint4*>(reinterpret_cast<char*>(vl[buf]) + at) = vs[e];
    }
  };

  // scores of a tile's 16 t + 4 lg + i in p[4 t + i], -inf where the lane's row does not see them
  auto scores = [&](int buf, int32_t x, uint32_t okc, float* p) {
    f32x4_t sc[2] = {zero4(), zero4()};
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Frag<T> k;
        k.load(kl[buf] + (16 * t + n) * RS + 32 * kk + 8 * lg);
        sc[t] = mma(k, qf[kk], sc[t]);
      }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 16 * t + 4 * lg + i;
        const int32_t j = sn.pos(x + key);
        const bool see = (((okc >> key) & 1) != 0) & (j <= tr) & ((j > tr - a.W) | (j < a.ns));
        p[4 * t + i] = see ? sc[t][i] * a.scale : -INFINITY;
      }
  };

  if (threadIdx.x == 0) any_bad = 0;
  __syncthreads();
  if (a.kn && blockIdx.y == 0) {
    const int32_t end = first_token(r0 + kSharedRows, a.G);
    append_rows<D * ES>(a, trow, g, tok0, p0, first_token(r0, a.G), end < ntok ? end : ntok);
  }
  if (v0 < v1) {
    fetch(v0, look(v0));
    Pages next = look(v0 + kPagedTile);
    uint32_t okc = there(v0);
    put(0, v0);
    int buf = 0;
    for (int32_t x = v0;; x += kPagedTile, buf ^= 1) {
      const bool more = x + kPagedTile < v1;
      uint32_t okn = 0;
      __syncthreads();
      if (more) {
        fetch(x + kPagedTile, next);
        next = look(x + 2 * kPagedTile);
        okn = there(x + kPagedTile);
      }
      if (sn.pos(x) <= tw1) {  // (a tile behind the wave's last row, in ascending order)
        float p[8];
        scores(buf, x, okc, p);
        float mx = m;
#pragma unroll
        for (int i = 0; i < 8; ++i) mx = fmaxf(mx, p[i]);
        mx = lg_max(mx);
        if (__any(mx > m)) {
          const float f = __builtin_amdgcn_exp2f(m - mx);
          m = mx;
          l *= f;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[ct][i] *= f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(p[i] - m);
          l += p[i];
        }
        Frag<T> pf;
        pf.set8(p);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          Frag<T> vc;
          load_colfrag2(vc, vl[buf], RS, 4 * lg, 16 + 4 * lg, 16 * ct);
          acc[ct] = mma(vc, pf, acc[ct]);
        }
      }
      if (!more) break;
      put(buf ^ 1, x + kPagedTile);
      okc = okn;
    }
    __syncthreads();
    if (any_bad) {
#pragma unroll 1
      for (int32_t x = v0; x < v1; x += kPagedTile) {
        if (!edge(x)) continue;
        fetch(x, look(x));
        const uint32_t okc = there(x);
        uint32_t rows = 0;
#pragma unroll
        for (int e = 0; e < NL; ++e)
          rows |= rows_of<LPR>(__ballot(!finite16(vs[e], T()))) << (RPI * e + wave * (64 / LPR));
        __syncthreads();
        if (lane == 0) bad[wave] = rows;
        put(0, x);
        __syncthreads();
        if (sn.pos(x) > tw1) continue;
        float p[8];
        scores(0, x, okc, p);
        uint32_t m4 = __builtin_amdgcn_readfirstlane(bad[0] | bad[1] | bad[2] | bad[3]);
        while (m4) {
          const int key = __builtin_ctz(m4);
          m4 &= m4 - 1;
          float w = -INFINITY;
#pragma unroll
          for (int i = 0; i < 8; ++i) w = i == ((key >> 4) * 4 + (key & 3)) ? p[i] : w;
          w = __shfl(__builtin_amdgcn_exp2f(w - m), ((key >> 2) & 3) * 16 + n);
          const int32_t j = sn.pos(x + key);
          const Slot sl = paged_slot(trow, j, a.shift, a.n_pages);
          const gptr_t vr = a.kn && j >= p0 ? (gptr_t)a.vn + ((tok0 + j - p0) * a.Hkv + g) * (D * ES)
                                            : (gptr_t)a.vp + slot_offset(a.vs, sl, g);
          if (!sees(a, j, tr)) continue;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            float y[4] = {acc[ct][0], acc[ct][1], acc[ct][2], acc[ct][3]};
            add_nonfinite4(y, vr + (16 * ct + 4 * lg) * ES, w, T());
            acc[ct] = f32x4_t{y[0], y[1], y[2], y[3]};
          }
        }
      }
    }
  }

  l = lg_sum(l);
  if (!rok) return;
  if (a.npiece > 1) {
    const int64_t rec = orow * a.npiece + blockIdx.y;
    if (lg == 0) {
      a.ml[rec * 2] = m;
      a.ml[rec * 2 + 1] = l;
    }
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
      *reinterpret_cast<float4*>(a.acc + rec * D + 16 * ct + 4 * lg) =
          make_float4(acc[ct][0], acc[ct][1], acc[ct][2], acc[ct][3]);
    return;
  }
  if (lg == 0) {
    const float lse2 = l > 0.f ? m + __builtin_amdgcn_logf(l) : l == 0.f ? -INFINITY : l;
    if (a.lse) a.lse[orow] = lse2 * kLn2;
    if (a.lse2) a.lse2[orow] = lse2;
  }
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

// The pieces of a row joined: a wave's lanes take the pieces'
// frames and sums (npiece <= 256, four each).  Bound by latency: 32 rows of 64
// pieces 3.6 us.
struct Joined {
  float M, L;
};
__device__ __forceinline__ float wave_max(float x) {
  x = dpp_max_row16(x);
  return lg_max(x);
}
__device__ __forceinline__ float wave_sum(float x) { return lg_sum(dpp_sum_rows<16>(x)); }

// f[u]: what piece lane + 64 u counts in the row's frame; -1: no part in it.
__device__ __forceinline__ Joined join_frames(const PagedArgs& a, int64_t r, float* f) {
  const int lane = threadIdx.x & 63;
  const float2* ml = reinterpret_cast<const float2*>(a.ml) + r * a.npiece;
  float2 x[kPagedMaxPieces / 64];
  Joined j = {kNoMax, 0.f};
#pragma unroll
  for (int u = 0; u < kPagedMaxPieces / 64; ++u) {
    x[u] = make_float2(kNoMax, 0.f);
    if (lane + 64 * u < a.npiece) x[u] = ml[lane + 64 * u];
    j.M = fmaxf(j.M, x[u].x);
  }
  j.M = wave_max(j.M);
#pragma unroll
  for (int u = 0; u < kPagedMaxPieces / 64; ++u) {
    // a piece without a part in the row has no acc either.  (Not one whose
    // factor underflows: infinities and NaN among its values show in the row
    // whatever their weight, as in a row of one piece.)
    f[u] = x[u].y == 0.f ? -1.f : __builtin_amdgcn_exp2f(x[u].x - j.M);
    j.L += x[u].y * f[u];
  }
  j.L = wave_sum(j.L);
  return j;
}
__device__ __forceinline__ float log2_sum(const Joined& j) {
  return j.L > 0.f ? j.M + __builtin_amdgcn_logf(j.L) : j.L == 0.f ? -INFINITY : j.L;
}

// Row r's output by NW waves (a workgroup's four, or one): each takes every
// NW-th piece, eight records at a time; their sums are added in order.
template <typename T, int D, int NW>
__device__ __forceinline__ void join_row(const PagedArgs& a, int64_t r, const Joined& j, const float* f,
                                         float (*part)[D]) {
  constexpr int E = D / 64;
  const int lane = threadIdx.x & 63, wave = NW == 1 ? 0 : threadIdx.x >> 6;
  const float* acc = a.acc + r * a.npiece * D + lane * E;
  float x[E] = {};
  for (int i0 = wave; i0 < a.npiece; i0 += 8 * NW) {
    float y[8][E], w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int p = i0 + NW * i;
      const float fu = p < 64 ? f[0] : p < 128 ? f[1] : p < 192 ? f[2] : f[3];
      w[i] = p < a.npiece ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(fu), p & 63)) : -1.f;
#pragma unroll
      for (int e = 0; e < E; ++e) y[i][e] = w[i] < 0.f ? 0.f : acc[int64_t(p) * D + e];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] += w[i] * y[i][e];
  }
  const float inv = j.L == 0.f ? 0.f : 1.f / j.L;
  if constexpr (NW == 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) reinterpret_cast<T*>(a.out)[r * D + lane * E + e] = from_f32<T>(x[e] * inv);
  } else {
    __syncthreads();
#pragma unroll
    for (int e = 0; e < E; ++e) part[wave][lane * E + e] = x[e];
    __syncthreads();
    if (int(threadIdx.x) < D) {
      const float y = part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x];
      reinterpret_cast<T*>(a.out)[r * D + threadIdx.x] = from_f32<T>(y * inv);
    }
  }
  if (lane == 0 && wave == 0) {
    const float lse2 = log2_sum(j);
    if (a.lse) a.lse[r] = lse2 * kLn2;
    if (a.lse2) a.lse2[r] = lse2;
  }
}

// NW waves per row: four where there are more than eight pieces (a wave's
// loads at once), else one, and four rows per workgroup.
template <typename T, int D, int NW>
__global__ __launch_bounds__(256) void paged_join(PagedArgs a, int64_t row0, int64_t rows) {
  __shared__ float part[4][D];
  int64_t r = int64_t(blockIdx.x) * (4 / NW);
  if constexpr (NW == 1) r += threadIdx.x >> 6;
  if (r >= rows) return;
  float f[kPagedMaxPieces / 64];
  const Joined j = join_frames(a, row0 + r, f);
  join_row<T, D, NW>(a, row0 + r, j, f, part);
}
template <typename T, int D>
hipError_t join_t(const PagedArgs& a, int64_t row0, int64_t rows, hipStream_t stream) {
  if (a.npiece > 8) paged_join<T, D, 4><<<uint32_t(rows), 256, 0, stream>>>(a, row0, rows);
  else paged_join<T, D, 1><<<uint32_t((rows + 3) / 4), 256, 0, stream>>>(a, row0, rows);
  return hipGetLastError();
}

// ---------------------------------------------------------------------------
// Decode: weights_j += sum over the group's heads of e^{s_j - lse}, from the
// raw scores that the attention left, and the rows' pieces joined in the same
// launch: of a (sequence, KV head) the first G workgroups join a row each, the
// others take 256 visible tokens each.  Bound by latency: the frames of the
// rows, then one read of the scores (asked for before the frames: no faster).
// 8 sequences, 64 / 8 heads, 8195 tokens each: 12 us.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_weights(PagedArgs a) {
  __shared__ float part[4][D], z[kMaxG];
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv;
  const int64_t row0 = int64_t(b) * a.Hq + g * a.G;
  float f[kPagedMaxPieces / 64];
  if (int(blockIdx.y) < a.G) {
    const Joined j = join_frames(a, row0 + blockIdx.y, f);
    join_row<T, D, 4>(a, row0 + blockIdx.y, j, f, part);
    return;
  }
#pragma unroll 1
  for (int h = threadIdx.x >> 6; h < a.G; h += 4) {
    const Joined j = join_frames(a, row0 + h, f);
    if ((threadIdx.x & 63) == 0) z[h] = log2_sum(j);
  }
  const int32_t len = seq_len(a, b);
  __syncthreads();
  if (len == 0) return;
  const Seen sn = seen_by(len - 1, len - 1, a.W, a.ns);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int32_t v0 = (blockIdx.y - a.G) * 256 + threadIdx.x;
#pragma unroll 1
  for (int64_t v = v0; v < sn.n; v += int64_t(gridDim.y - a.G) * 256) {
    const int32_t j = sn.pos(int32_t(v));
    const Slot sl = paged_slot(trow, j, a.shift, a.n_pages);
    float s[kMaxG];
#pragma unroll
    for (int h = 0; h < kMaxG; ++h) s[h] = h < a.G ? a.scores[(row0 + h) * a.nv + v] : 0.f;
    if (!sl.ok) continue;
    float* at = a.wp + ((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot;
    const float w = *at;
    float y = 0.f;
#pragma unroll
    for (int h = 0; h < kMaxG; ++h)
      if (h < a.G && z[h] != -INFINITY) y += __builtin_amdgcn_exp2f(s[h] - z[h]);
    *at = w + y;
  }
}

// Prefill: the last n_observe queries of each sequence.  A wave owns 32 keys
// (their K fragments in registers) and goes through the scored rows in order,
// 64 at a time through LDS: no sum's order depends on timing.  Bound by the
// latency of its loads where few rows are scored, else by its products and
// exponentials.  32 queries of 4 heads over 4036 tokens, 8 sequences of 8 KV
// heads: 32 us (K again: 13 at 5 TB/s).
template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_weights(PagedArgs a, PagedSeqs s, int n_observe) {
  constexpr int KK = D / 32, ES = int(sizeof(T)), RS = D + 16 / ES, NB = 64;  // rows of a block
  constexpr int P = D * ES / 16, NP = NB * P / 256;                           // 16-byte pieces of a row, of a thread
  __shared__ __align__(16) T qs[NB * RS];
  __shared__ float zs[NB];
  __shared__ int32_t ts[NB];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, lg = lane >> 4;
  const int i = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, b = s.seq0 + i;
  const int32_t len = seq_len(a, b), ntok = s.len[i], p0 = len - ntok;
  const int32_t obs = ntok < n_observe ? ntok : n_observe;
  if (len == 0 || obs == 0) return;
  const int32_t first = ntok - obs;  // first scored token
  const int32_t t0 = p0 + first > 0 ? p0 + first : 0;
  const Seen sn = seen_by(t0, len - 1, a.W, a.ns);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const int32_t row0 = first * a.G, rows = obs * a.G;
  uint4 st[NP];
  auto fetch = [&](int32_t rb) {  // 64 rows of q
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      const int32_t x = rb + (e * 256 + int(threadIdx.x)) / P, r = row0 + (x < rows ? x : rows - 1);
      const int64_t orow = (int64_t(s.start[i]) + r / a.G) * a.Hq + g * a.G + r % a.G;
      st[e] = gload16<false>((gptr_t)a.q + orow * (D * ES) + (threadIdx.x % P) * 16);
    }
  };
  for (int32_t x0 = blockIdx.y * 128; x0 < sn.n; x0 += int32_t(gridDim.y) * 128) {
    const int32_t x = x0 + wave * 32;
    fetch(0);
    Frag<T> kf[2][KK];
    uint32_t ok[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int32_t vi = x + 16 * t + n;
      Slot sl = {0, 0, false};
      if (vi < sn.n) sl = paged_slot(trow, sn.pos(vi), a.shift, a.n_pages);
      ok[t] = uint32_t(__ballot(sl.ok)) & 0xffffu;
      const gptr_t kr = sl.ok ? (gptr_t)a.kp + slot_offset(a.ks, sl, g) : (gptr_t)zero_row;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) gload_frag<false>(kf[t][kk], kr + (32 * kk + 8 * lg) * ES);
    }
    // positions of this lane's keys; not there: behind every query
    int32_t j[2][4];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        j[t][e] = (ok[t] >> (4 * lg + e)) & 1 ? sn.pos(x + 16 * t + 4 * lg + e) : 0x7fffffff;
    float w[2][4] = {};
    for (int32_t rb = 0; rb < rows; rb += NB) {
      __syncthreads();  // the block before is read
#pragma unroll
      for (int e = 0; e < NP; ++e) {
        const int at = e * 256 + int(threadIdx.x);
        *reinterpret_cast<uint4*>(reinterpret_cast<char*>(qs + (at / P) * RS) + (at % P) * 16) = st[e];
      }
      if (threadIdx.x < NB) {
        const int32_t y = rb + int(threadIdx.x), r = row0 + (y < rows ? y : rows - 1);
        const float z = a.lse2[(int64_t(s.start[i]) + r / a.G) * a.Hq + g * a.G + r % a.G];
        zs[threadIdx.x] = z;
        ts[threadIdx.x] = y < rows && z != -INFINITY ? p0 + r / a.G : -1;  // -1: sees nothing
      }
      __syncthreads();
      if (rb + NB < rows) fetch(rb + NB);
      const int tiles = (rows - rb < NB ? rows - rb + 15 : NB) / 16;
      for (int rt = 0; rt < tiles; ++rt) {
        f32x4_t sc[2] = {zero4(), zero4()};
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
          Frag<T> qf;
          qf.load(qs + (16 * rt + n) * RS + 32 * kk + 8 * lg);
#pragma unroll
          for (int t = 0; t < 2; ++t) sc[t] = mma(kf[t][kk], qf, sc[t]);
        }
        const float z = zs[16 * rt + n];
        const int32_t tr = ts[16 * rt + n];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const bool see = (j[t][e] <= tr) & ((j[t][e] > tr - a.W) | (j[t][e] < a.ns));
            const float y = __builtin_amdgcn_exp2f(sc[t][e] * a.scale - z);
            w[t][e] += see ? y : 0.f;
          }
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = dpp_sum_rows<16>(w[t][e]);
        if (n == 0 && j[t][e] != 0x7fffffff) {
          const Slot sl = paged_slot(trow, j[t][e], a.shift, a.n_pages);
          a.wp[((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot] += y;
        }
      }
  }
}

template <typename T, int D>
hipError_t decode_t(const PagedArgs& a, int64_t keys, hipStream_t stream) {
  attend_rows<T, D, NoSeqs><<<dim3(a.B * a.Hkv, a.npiece), 256, 0, stream>>>(a, NoSeqs());
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.scores) {
    const int64_t chunks = std::min<int64_t>((keys + 255) / 256, 32768);
    join_weights<T, D><<<dim3(a.B * a.Hkv, uint32_t(a.G + chunks)), 256, 0, stream>>>(a);
  } else if (a.npiece > 1) {
    return join_t<T, D>(a, 0, int64_t(a.B) * a.Hq, stream);
  }
  return hipGetLastError();
}

template <typename T, int D>
hipError_t prefill_t(const PagedArgs& a, const PagedSeqs& s, int tile_rows, hipStream_t stream) {
  const int64_t tiles = s.tile0[s.nseq];
  if (tiles == 0) return hipSuccess;
  const dim3 grid(uint32_t(tiles * a.Hkv), a.npiece);
  if constexpr (sizeof(T) == 2) {
    if (tile_rows == kTileRows) attend_tiles<D><<<grid, 256, 0, stream>>>(a, s);
  }
  if (tile_rows == kSharedRows) attend_shared<T, D><<<grid, 256, 0, stream>>>(a, s);
  else if (tile_rows == kPagedRows) attend_rows<T, D, PagedSeqs><<<grid, 256, 0, stream>>>(a, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.npiece == 1) return e;
  const int64_t row0 = int64_t(s.start[0]) * a.Hq;
  const int64_t rows = (int64_t(s.start[s.nseq - 1]) + s.len[s.nseq - 1]) * a.Hq - row0;
  return join_t<T, D>(a, row0, rows, stream);
}

}  // namespace

hipError_t launch_paged_decode(const PagedArgs& a, int64_t keys, int d, int dtype, hipStream_t stream) {
  if (dtype == GLIDE_BF16)
    return d == 128 ? decode_t<bf16_t, 128>(a, keys, stream) : decode_t<bf16_t, 64>(a, keys, stream);
  return d == 128 ? decode_t<float, 128>(a, keys, stream) : decode_t<float, 64>(a, keys, stream);
}

hipError_t launch_paged_prefill(const PagedArgs& a, const PagedSeqs& s, int d, int dtype, int tile_rows,
                                hipStream_t stream) {
  if (dtype == GLIDE_BF16)
    return d == 128 ? prefill_t<bf16_t, 128>(a, s, tile_rows, stream) : prefill_t<bf16_t, 64>(a, s, tile_rows, stream);
  return d == 128 ? prefill_t<float, 128>(a, s, tile_rows, stream) : prefill_t<float, 64>(a, s, tile_rows, stream);
}

hipError_t launch_paged_join(const PagedArgs& a, int64_t row0, int64_t rows, int d, int dtype, hipStream_t stream) {
  if (dtype == GLIDE_BF16)
    return d == 128 ? join_t<bf16_t, 128>(a, row0, rows, stream) : join_t<bf16_t, 64>(a, row0, rows, stream);
  return d == 128 ? join_t<float, 128>(a, row0, rows, stream) : join_t<float, 64>(a, row0, rows, stream);
}

hipError_t launch_paged_weights(const PagedArgs& a, const PagedSeqs& s, int n_observe, int64_t keys, int d, int dtype,
                                hipStream_t stream) {
  const dim3 grid(s.nseq * a.Hkv, uint32_t(std::min<int64_t>((keys + 127) / 128, 4096)));
  if (dtype == GLIDE_BF16) {
    if (d == 128) prefill_weights<bf16_t, 128><<<grid, 256, 0, stream>>>(a, s, n_observe);
    else prefill_weights<bf16_t, 64><<<grid, 256, 0, stream>>>(a, s, n_observe);
  } else {
    if (d == 128) prefill_weights<float, 128><<<grid, 256, 0, stream>>>(a, s, n_observe);
    else prefill_weights<float, 64><<<grid, 256, 0, stream>>>(a, s, n_observe);
  }
  return hipGetLastError();
}

}  // namespace glide
