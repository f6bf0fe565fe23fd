// Softmax attention over a paged cache held in 4 bits: sliding window, sinks,
// grouped query heads, pieces of long rows.  The cache's values are bf16
// numbers, so bf16 matrix instructions take them without rounding; fp32 queries
// and weights go in as three bf16 parts each (8 bits of 24), whose products are
// exact and summed in fp32.
#include <type_traits>

#include "nibble.h"

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
__device__ __forceinline__ void wave_lds_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}
__device__ __forceinline__ int32_t seq_len(const PagedArgs& a, int b) {
  const int32_t n = a.lens[b];
  return n < 0 ? 0 : n > a.cap ? a.cap : n;
}

// Eight numbers as bf16 operands: one rounded (bf16 calls: half a step, 2^-8 of
// each at most), or three parts that sum to each exactly (fp32 calls: what is
// left after 24 bits is 0; bits below 2^-133 have no place).
template <typename T>
struct Parts {
  static constexpr int N = sizeof(T) == 2 ? 1 : 3;
  Frag<bf16_t> f[N];
  __device__ __forceinline__ void set8(const float* x) {
    split8(x, [](Frag<bf16_t>& part, const float* y) { part.set8(y); });
  }
  // The largest fp32 numbers would round to infinity: a query's parts are cut off.
  __device__ __forceinline__ void load(const T* p) {
    Frag<T> x;
    x.load(p);
    if constexpr (N == 1) {
      f[0] = x;
    } else {
      split8(x.v, [](Frag<bf16_t>& part, const float* y) {
        auto upper = [](float a, float b) {  // their upper halves, a's in the lower
          return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
        };
        part.v = make_uint4(upper(y[0], y[1]), upper(y[2], y[3]), upper(y[4], y[5]), upper(y[6], y[7]));
      });
    }
  }
  template <typename F>  // part(f, y): y to the operand f
  __device__ __forceinline__ void split8(const float* x, F part) {
    part(f[0], x);
    if constexpr (N == 3) {
      float y[8], z[8];
      f[0].to_floats(y);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i] - y[i];
      part(f[1], y);
      f[1].to_floats(z);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = y[i] - z[i];
      part(f[2], z);
    }
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i].zero();
  }
};
template <typename T>
__device__ __forceinline__ f32x4_t mma_parts(const Frag<bf16_t>& a, const Parts<T>& b, f32x4_t c) {
#pragma unroll
  for (int i = Parts<T>::N - 1; i >= 0; --i) c = mma(a, b.f[i], c);  // the small parts first
  return c;
}

// W bytes at p (4-byte aligned), non-temporal where a decode call reads rows once.
template <bool NT, int W>
__device__ __forceinline__ void gload_words(uint32_t* x, gptr_t p) {
  typedef uint32_t vec_t __attribute__((ext_vector_type(W / 4)));
  const auto q = (const vec_t __attribute__((address_space(1)))*)p;
  vec_t v;
  if constexpr (NT) v = __builtin_nontemporal_load(q);
  else v = *q;
#pragma unroll
  for (int i = 0; i < W / 4; ++i) x[i] = v[i];
}

// ---------------------------------------------------------------------------
// Attention of one tile of 16 rows ((token, head) pairs of one KV head) over
// one piece of the tokens that they see; the four waves take tiles of 64 keys
// in turn, each with a running maximum and sum of its own, joined at the end.
//   S^T = K Q^T: a lane reads a quarter of a key's codes (one scale), which are,
//   converted, its operands of the products as they stand: the elements of a
//   slab are summed in the order 8 s + (d/4) g + 0..7 for slab s and lane group
//   g, of the queries alike.  O^T += V^T P^T with keys in the order 4 g + 0..3,
//   16 + 4 g + 0..3; V goes through LDS, converted, for its columns.
// A row that is not there is read as row 0 of the pools: every code is a finite
// number, and weights of 0 leave it out.
// Bound by HBM in long decodes (bf16, d = 128): 32 sequences of 16K .. 32K
// tokens, 8 KV heads, 856 MB in 152 us (5.6 TB/s; the same loads with nothing
// done to them: 150); the conversions take half of the vector cycles.  Smaller
// calls are bound by the chain table -> rows -> scores -> join.
// The scaled matrix instruction would take the codes of K as they are, with q
// in two fp8 parts, but its sums over 128 products are off by 2^-17 of their
// terms; bf16 products are summed in fp32.
struct NoSeqs {};
template <typename T, int D, typename Seqs, int TK>  // Seqs: PagedSeqs, or NoSeqs for a decode call; TK: keys of a tile
__global__ __launch_bounds__(256, TK == 32 ? 4 : 2) void nibble_rows(PagedArgs a, Pools4 pools, Seqs s) {
  constexpr bool DECODE = std::is_same<Seqs, NoSeqs>::value;
  constexpr int KK = D / 32, CT = D / 16, EPL = D / 4, W = EPL / 2, NW = W / 4, RS = D + 16;
  constexpr int ST = TK / 16;  // sub-tiles of 16 keys
  __shared__ __align__(16) bf16_t vlds[4][TK * RS];
  __shared__ float sm[4][16], sl_[4][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, lg = lane >> 4;
  int b, g, r0, ntok;
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
  const int nrow = ntok * a.G;
  const int32_t len = seq_len(a, b), p0 = len - ntok;
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
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;

  Parts<T> qf[KK];
#pragma unroll
  for (int kk = 0; kk < KK; ++kk) {
    qf[kk].load(reinterpret_cast<const T*>(a.q) + orow * D + EPL * lg + 8 * kk);
    if (!rok) qf[kk].zero();
    if (a.scale < 0) {  // scores of -q: the frame is a maximum of raw scores
#pragma unroll
      for (int x = 0; x < Parts<T>::N; ++x) qf[kk].f[x].negate();
    }
  }
  const float c = fabsf(a.scale);
  float m = kNoMax, l = 0.f;
  f32x4_t acc[CT];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) acc[ct] = zero4();
  bf16_t* vt = vlds[wave];

  // A tile's rows are asked for as soon as the one before it is out of the
  // registers, its page numbers a tile earlier.  Lane x looks up key x.
  struct At {
    int32_t j, page;  // position (-1: behind the piece) and page
  };
  auto look = [&](int32_t x) {
    At p;
    const int32_t vi = x + (lane & (TK - 1));
    p.j = vi < v1 ? sn.pos(vi) : -1;
    p.page = trow[(vi < v1 ? p.j : 0) >> a.shift];
    return p;
  };
  // Scales of a tile in one load: lane x has those of key x % 32 (K in the lower
  // half of the wave, V in the upper), all of its row.
  constexpr int SB = D / kGroup4;  // bytes
  uint32_t kc[ST][NW], vc[ST][NW], sc8[ST / 2];
  uint64_t okm = 0;  // the tile's rows that are there
  auto fetch = [&](const At& p) {
    const bool good = p.j >= 0 && uint32_t(p.page) < uint32_t(a.n_pages);
    okm = __ballot(good) | (TK == 64 ? 0 : ~uint64_t(0) << (TK & 63));
    // (row numbers fit 32 bits: checked on the host)
    const uint32_t row = good ? ((uint32_t(p.page) * uint32_t(a.Hkv) + uint32_t(g)) << a.shift) +
                                    uint32_t(p.j & ((1 << a.shift) - 1))
                              : 0u;
#pragma unroll
    for (int u = 0; u < ST / 2; ++u) {
      const uint64_t rt = TK == 32 ? row : uint32_t(__shfl(int(row), 32 * u + (lane & 31)));
      const gptr_t at = (gptr_t)(lane < 32 ? pools.ks : pools.vs) + rt * SB;
      if constexpr (SB == 4) sc8[u] = *(const uint32_t __attribute__((address_space(1)))*)at;
      else sc8[u] = *(const uint16_t __attribute__((address_space(1)))*)at;
    }
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      const uint64_t rt = uint32_t(__shfl(int(row), 16 * t + n)), at = rt * (D / 2) + lg * W;
      gload_words<DECODE, W>(kc[t], (gptr_t)pools.kc + at);
      gload_words<DECODE, W>(vc[t], (gptr_t)pools.vc + at);
    }
  };
  const int sbit = 8 * ((lg * EPL) / kGroup4);  // the lane's group among a row's scales

  constexpr int STEP = 4 * TK;
  int32_t x = v0 + wave * TK;
  At next = {};
  if (x < v1) {
    const At first = look(x);
    next = look(x + STEP);
    fetch(first);
  }
  for (; x < v1; x += STEP) {
    f32x4_t sc[ST];
    const uint64_t okc = okm;
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      const uint32_t ks = (uint32_t(__shfl(int(sc8[t / 2]), 16 * (t & 1) + n)) >> sbit) & 255u;
      const uint32_t vs = (uint32_t(__shfl(int(sc8[t / 2]), 32 + 16 * (t & 1) + n)) >> sbit) & 255u;
      sc[t] = zero4();
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        Frag<bf16_t> k;
        k.v = bf16_of_codes(kc[t][kk], scale_of(ks));
        sc[t] = mma_parts<T>(k, qf[kk], sc[t]);
        *reinterpret_cast<uint4*>(vt + (16 * t + n) * RS + EPL * lg + 8 * kk) = bf16_of_codes(vc[t][kk], scale_of(vs));
      }
    }
    if (x + STEP < v1) {
      const At now = next;
      next = look(x + 2 * STEP);
      fetch(now);
    }
    // what a row does not see (tested for the wave: few tiles hold any)
    if constexpr (DECODE) {
      if (~okc) {
#pragma unroll
        for (int t = 0; t < ST; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!((okc >> (16 * t + 4 * lg + i)) & 1)) sc[t][i] = -INFINITY;
      }
    } else {
#pragma unroll
      for (int t = 0; t < ST; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int key = 16 * t + 4 * lg + i;
          const int32_t j = sn.pos(x + key);
          if (!((okc >> key) & 1) || j > tr || (j <= tr - a.W && j >= a.ns)) sc[t][i] = -INFINITY;
        }
    }
    // the frame moves only when a score passes it by 2^8: weights up to that
    // round alike, and fp32 sums hold them
    float mx = sc[0][0];
#pragma unroll
    for (int t = 0; t < ST; ++t)
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
    float p[4 * ST];
#pragma unroll
    for (int i = 0; i < 4 * ST; ++i) {
      p[i] = __builtin_amdgcn_exp2f(fmaf(sc[i >> 2][i & 3], c, -m));
      l += p[i];
    }
    Parts<T> pf[ST / 2];
#pragma unroll
    for (int u = 0; u < ST / 2; ++u) pf[u].set8(p + 8 * u);
    wave_lds_order();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int u = 0; u < ST / 2; ++u) {
        Frag<bf16_t> v;
        load_colfrag2(v, vt + 32 * u * RS, RS, 4 * lg, 16 + 4 * lg, 16 * ct);
        acc[ct] = mma_parts<T>(v, pf[u], acc[ct]);
      }
    }
    wave_lds_order();
  }

  // the four waves' parts: each row's frame, then the sums in it
  l = lg_sum(l);
  if (lane < 16) {
    sm[wave][lane] = m;
    sl_[wave][lane] = l;
  }
  __syncthreads();
  float M = kNoMax;
#pragma unroll
  for (int w = 0; w < 4; ++w) M = fmaxf(M, sm[w][n]);
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
  if (a.npiece > 1) {
    const int64_t rec = o2 * a.npiece + blockIdx.y;
    if (e0 == 0) {
      a.ml[rec * 2] = Mr;
      a.ml[rec * 2 + 1] = Lr;
    }
#pragma unroll
    for (int e = 0; e < D / 16; ++e) a.acc[rec * D + e0 + e] = red[rr * RD + e0 + e];
  } else {
    if (e0 == 0 && a.lse) a.lse[o2] = (Lr > 0.f ? Mr + __builtin_amdgcn_logf(Lr) : Lr == 0.f ? -INFINITY : Lr) * kLn2;
    const float inv = Lr == 0.f ? 0.f : 1.f / Lr;
    T* w = reinterpret_cast<T*>(a.out) + o2 * D + e0;
#pragma unroll
    for (int e = 0; e < D / 16; ++e) w[e] = from_f32<T>(red[rr * RD + e0 + e] * inv);
  }
}

// ---------------------------------------------------------------------------
// Attention of many rows: a workgroup takes WAVES * 32 rows ((token, head) pairs
// of one KV head, 32 per wave) over the 64-key tiles that any of them sees; a
// tile's codes are converted once for the workgroup, on their way into LDS.
//   S^T = K Q^T with 32x32x16 MFMAs: a lane holds the scores of one row, 16 of
//   each 32 keys, in the order that the right operand of O^T += V^T P^T takes
//   (keys 8j + 4h + 0..3 of lane half h), so the weights never leave its
//   registers; V^T comes from the transposing LDS reads.
//   Row sums of the weights are taken before they are rounded (bf16): lse is
//   exact to fp32.  The frame (a row's maximum) moves only when a score passes
//   it by 2^8: weights up to 2^8 round alike, and fp32 sums hold them.
// A 16-byte piece c of row r is kept at piece c ^ swz(r) of the row: eight
// consecutive rows' pieces, and four rows' 64-byte V segments, lie in different
// banks.
template <int D>
__device__ __forceinline__ int swz(int r) {
  return D == 128 ? ((r & 3) << 2) | ((r >> 2) & 3) : (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
}
typedef float f32x16_t __attribute__((ext_vector_type(16)));
template <typename T>
__device__ __forceinline__ f32x16_t mma32_parts(uint4 a, const Parts<T>& b, f32x16_t c) {
#pragma unroll
  for (int i = Parts<T>::N - 1; i >= 0; --i)
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b.f[i].v),
                                                c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ uint4 vt_frag(const char* p, const char* q) {
  const i16x4_t a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(__attribute__((address_space(3))) char*)p);
  const i16x4_t b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)(__attribute__((address_space(3))) char*)q);
  const uint2 x = __builtin_bit_cast(uint2, a), y = __builtin_bit_cast(uint2, b);
  return make_uint4(x.x, x.y, y.x, y.y);
}

template <typename T, int D, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 8 ? 2 : Parts<T>::N == 1 ? 2 : 1) void nibble_tiles(PagedArgs a, Pools4 pools,
                                                                                  PagedSeqs s) {
  constexpr int KK = D / 16, CT = D / 32, RB = 2 * D, ROWS = 32 * WAVES, NS = Parts<T>::N;
  constexpr int KB = kTileKeys * RB;  // bytes of a K (or V) tile in LDS
  // staging: thread (row, part): of a row, PT parts of EPT elements each (W bytes of codes)
  constexpr int PT = WAVES, EPT = D / PT, W = EPT / 2, NW = W / 4;
  __shared__ __align__(16) char lds[2][2 * KB];
  __shared__ uint32_t there[2][4];  // rows of a tile that have a page, 16 bits each
  const int lane = threadIdx.x & 63, h = lane >> 5, q = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int tile = s.tile0[s.nseq] - 1 - int(blockIdx.x) / a.Hkv, g = int(blockIdx.x) % a.Hkv;
  const int si = find_seq(s, tile), b = s.seq0 + si, ntok = s.len[si];
  const int32_t len = __builtin_amdgcn_readfirstlane(seq_len(a, b)), p0 = len - ntok;
  const int r0 = (tile - s.tile0[si]) * ROWS, rend = ntok * a.G;
  const int rlast = r0 + ROWS < rend ? r0 + ROWS - 1 : rend - 1;
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

  Parts<T> qf[KK];
  {
    const T* qp = reinterpret_cast<const T*>(a.q) + orow * D + 8 * h;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {
      qf[kk].load(qp + 16 * kk);
      if (!rok) qf[kk].zero();
      if (a.scale < 0) {  // scores of -q: the frame is a maximum of raw scores
#pragma unroll
        for (int x = 0; x < NS; ++x) qf[kk].f[x].negate();
      }
    }
  }
  const float c = fabsf(a.scale);

  // staging: 16 rows to 16 neighbouring lanes, so that eight lanes' pieces lie in different banks
  const int srow = (threadIdx.x & 15) + 16 * (wave & 3), part = (wave >> 2) * 4 + (lane >> 4);
  auto page_of = [&](int32_t i) {
    const int32_t at = (key0(i) + srow) >> a.shift;
    return trow[at < last_entry ? at : last_entry];
  };
  struct Stage {
    uint32_t k[NW], v[NW], ks, vs;
    uint32_t there;
  };
  auto fetch = [&](int32_t i, int32_t page, Stage& st) {
    const bool ok = uint32_t(page) < uint32_t(a.n_pages);
    st.there = uint32_t(__ballot(ok)) & 0xffffu;
    // (row numbers fit 32 bits: checked on the host; a row that is not there is read as row 0, and masked)
    const uint64_t row = ok ? ((uint32_t(page) * uint32_t(a.Hkv) + uint32_t(g)) << a.shift) +
                                  uint32_t((key0(i) + srow) & ((1 << a.shift) - 1))
                            : 0u;
    const uint64_t at = row * (D / 2) + part * W, sc = row * (D / kGroup4) + (part * EPT) / kGroup4;
    gload_words<false, W>(st.k, (gptr_t)pools.kc + at);
    gload_words<false, W>(st.v, (gptr_t)pools.vc + at);
    st.ks = pools.ks[sc];
    st.vs = pools.vs[sc];
  };
  auto put = [&](int at, const Stage& st) {
    const float ks = scale_of(st.ks), vs = scale_of(st.vs);
    char* w = lds[at] + srow * RB;
    const int sw = swz<D>(srow);
#pragma unroll
    for (int x = 0; x < NW; ++x) {
      const int o = ((part * NW + x) ^ sw) << 4;
      *reinterpret_cast<uint4*>(w + o) = bf16_of_codes(st.k[x], ks);
      *reinterpret_cast<uint4*>(w + KB + o) = bf16_of_codes(st.v[x], vs);
    }
    if (wave < 4 && lane == 0) there[at][wave] = st.there;
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
  auto masks = [&](int32_t k0, const uint32_t* okp, f32x16_t* sc) {
    // what the rows do not see, where the tile may hold any (each kind tested
    // for the wave): keys after a row, keys before its window that are no
    // sinks, keys whose page is not there
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
    if ((okp[0] & okp[1] & okp[2] & okp[3]) != 0xffffu) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint32_t m = (okp[2 * t] | okp[2 * t + 1] << 16) >> (4 * h);
#pragma unroll
        for (int e = 0; e < 16; ++e) sc[t][e] = (m >> (8 * (e >> 2) + (e & 3))) & 1 ? sc[t][e] : -INFINITY;
      }
    }
  };
  auto compute = [&](int at, int32_t i) {
    const char* buf = lds[at];
    const int32_t k0 = key0(i);
    if (k0 > tw1 || (k0 + kTileKeys <= tw0 - a.W + 1 && k0 >= a.ns)) return;  // nothing for this wave
    f32x16_t sc[2];
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[t][e] = 0.f;
#pragma unroll
    for (int kk = 0; kk < KK; ++kk)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const uint4 kf = *reinterpret_cast<const uint4*>(buf + klane + 32 * t * RB + (((2 * kk) ^ ksw) << 4));
        sc[t] = mma32_parts<T>(kf, qf[kk], sc[t]);
      }
    if constexpr (NS == 1) {
      __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
      for (int u = 0; u < KK - 3; ++u) {
        __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, 6, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    auto vfrag = [&](int sl, int ct) {
      const char* p = buf + vlane + 16 * sl * RB + (((4 * ct) ^ vsw) << 4);
      const char* p2 = buf + vlane + (16 * sl + 8) * RB + (((4 * ct) ^ vsw ^ 2) << 4);
      return vt_frag(p, p2);
    };
    uint4 vf[CT];
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) vf[ct] = vfrag(0, ct);
    uint32_t okp[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) okp[x] = __builtin_amdgcn_readfirstlane(there[at][x]);
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
    float pw[8];
    auto weights2 = [&](int sl, int e) {  // elements e, e + 1 of slab sl
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const float y = __builtin_amdgcn_exp2f(fmaf(sc[sl >> 1][8 * (sl & 1) + e + x], c, -mc));
        l += y;
        pw[e + x] = y;
      }
    };
#pragma unroll
    for (int e = 0; e < 4; ++e) weights2(0, 2 * e);
    Parts<T> pf;
    pf.set8(pw);
#pragma unroll
    for (int sl = 0; sl < 4; ++sl) {
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        if constexpr (NS == 1) __builtin_amdgcn_sched_barrier(0);
        o[ct] = mma32_parts<T>(vf[ct], pf, o[ct]);
        if (sl < 3) {
          vf[ct] = vfrag(sl + 1, ct);
#pragma unroll
          for (int e = 0; e < 4 / CT; ++e) weights2(sl + 1, 2 * (ct * (4 / CT) + e));
        }
      }
      if (sl < 3) pf.set8(pw);
    }
    if constexpr (NS == 1) __builtin_amdgcn_sched_barrier(0);
  };

  if (i0 < i1) {
    Stage st;
    fetch(i0, page_of(i0), st);
    int32_t page = page_of(i0 + 1 < i1 ? i0 + 1 : i0);
    put(0, st);
    for (int32_t i = i0;; ++i) {
      const int cur = (i - i0) & 1;
      __syncthreads();
      if (i + 1 < i1) {
        fetch(i + 1, page, st);
        page = page_of(i + 2 < i1 ? i + 2 : i + 1);
      }
      compute(cur, i);
      if (i + 1 >= i1) break;
      put(cur ^ 1, st);
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
  if (rok && h == 0 && a.lse)
    a.lse[orow] = (l > 0.f ? mc + __builtin_amdgcn_logf(l) : l == 0.f ? -INFINITY : l) * kLn2;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if constexpr (NS == 1) {
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
  } else if (rok) {
    float* w = reinterpret_cast<float*>(a.out) + orow * D + 4 * h;
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<float4*>(w + 32 * ct + 8 * e) =
            make_float4(o[ct][4 * e] * inv, o[ct][4 * e + 1] * inv, o[ct][4 * e + 2] * inv, o[ct][4 * e + 3] * inv);
  }
}

template <typename T, int D>
hipError_t decode_t(const PagedArgs& a, const Pools4& p, int tile_keys, hipStream_t stream) {
  const dim3 grid(a.B * a.Hkv, a.npiece);
  if (tile_keys == 64) {
    nibble_rows<T, D, NoSeqs, 64><<<grid, 256, 0, stream>>>(a, p, NoSeqs());
    return hipGetLastError();
  }
  if constexpr (sizeof(T) == 2) {
    if (tile_keys == 32) {
      nibble_rows<T, D, NoSeqs, 32><<<grid, 256, 0, stream>>>(a, p, NoSeqs());
      return hipGetLastError();
    }
  }
  return hipErrorInvalidValue;  // no such kernel
}
template <typename T, int D>
hipError_t prefill_t(const PagedArgs& a, const Pools4& p, const PagedSeqs& s, int tile_rows, hipStream_t stream) {
  const dim3 grid(uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv), a.npiece);
  if (tile_rows == kRows4Big) nibble_tiles<T, D, 8><<<grid, 512, 0, stream>>>(a, p, s);
  else if (tile_rows == kRows4) nibble_tiles<T, D, 4><<<grid, 256, 0, stream>>>(a, p, s);
  else if (tile_rows == kPagedRows) nibble_rows<T, D, PagedSeqs, 64><<<grid, 256, 0, stream>>>(a, p, s);
  else return hipErrorInvalidValue;  // no such kernel
  return hipGetLastError();
}

}  // namespace

hipError_t launch_nibble_decode(const PagedArgs& a, const Pools4& p, int d, int dtype, int tile_keys,
                                hipStream_t stream) {
  hipError_t e;
  if (dtype == GLIDE_BF16)
    e = d == 128 ? decode_t<bf16_t, 128>(a, p, tile_keys, stream) : decode_t<bf16_t, 64>(a, p, tile_keys, stream);
  else
    e = d == 128 ? decode_t<float, 128>(a, p, tile_keys, stream) : decode_t<float, 64>(a, p, tile_keys, stream);
  if (e != hipSuccess || a.npiece == 1) return e;
  return launch_paged_join(a, 0, int64_t(a.B) * a.Hq, d, dtype, stream);
}

hipError_t launch_nibble_prefill(const PagedArgs& a, const Pools4& p, const PagedSeqs& s, int d, int dtype,
                                 int tile_rows, hipStream_t stream) {
  if (s.tile0[s.nseq] == 0) return hipSuccess;
  hipError_t e;
  if (dtype == GLIDE_BF16)
    e = d == 128 ? prefill_t<bf16_t, 128>(a, p, s, tile_rows, stream) : prefill_t<bf16_t, 64>(a, p, s, tile_rows, stream);
  else
    e = d == 128 ? prefill_t<float, 128>(a, p, s, tile_rows, stream) : prefill_t<float, 64>(a, p, s, tile_rows, stream);
  if (e != hipSuccess || a.npiece == 1) return e;
  const int64_t row0 = int64_t(s.start[0]) * a.Hq;
  const int64_t rows = (int64_t(s.start[s.nseq - 1]) + s.len[s.nseq - 1]) * a.Hq - row0;
  return launch_paged_join(a, row0, rows, d, dtype, stream);
}

}  // namespace glide
