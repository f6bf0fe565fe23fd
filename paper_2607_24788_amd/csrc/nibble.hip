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
// left after 24 bits is 0).
template <typename T>
struct Parts {
  static constexpr int N = sizeof(T) == 2 ? 1 : 3;
  Frag<bf16_t> f[N];
  __device__ __forceinline__ void set8(const float* x) {
    f[0].set8(x);
    if constexpr (N == 3) {
      float y[8], z[8];
      f[0].to_floats(y);
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = x[i] - y[i];
      f[1].set8(y);
      f[1].to_floats(z);
#pragma unroll
      for (int i = 0; i < 8; ++i) z[i] = y[i] - z[i];
      f[2].set8(z);
    }
  }
  __device__ __forceinline__ void load(const T* p) {
    Frag<T> x;
    x.load(p);
    if constexpr (N == 1) {
      f[0] = x;
    } else {
      set8(x.v);
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
struct NoSeqs {};
constexpr int kTile4 = 64;
template <typename T, int D, typename Seqs>  // Seqs: PagedSeqs, or NoSeqs for a decode call
__global__ __launch_bounds__(256, 2) void nibble_rows(PagedArgs a, Pools4 pools, Seqs s) {
  constexpr bool DECODE = std::is_same<Seqs, NoSeqs>::value;
  constexpr int KK = D / 32, CT = D / 16, EPL = D / 4, W = EPL / 2, NW = W / 4, RS = D + 16;
  __shared__ __align__(16) bf16_t vlds[4][kTile4 * RS];
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
  }
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
    const int32_t vi = x + lane;
    p.j = vi < v1 ? sn.pos(vi) : -1;
    p.page = trow[(vi < v1 ? p.j : 0) >> a.shift];
    return p;
  };
  uint32_t kc[4][NW], vc[4][NW], ks[4], vs[4];
  uint64_t okm = 0;  // the tile's rows that are there
  auto fetch = [&](const At& p) {
    const bool good = p.j >= 0 && uint32_t(p.page) < uint32_t(a.n_pages);
    okm = __ballot(good);
    // (row numbers fit 32 bits: checked on the host)
    const uint32_t row = good ? ((uint32_t(p.page) * uint32_t(a.Hkv) + uint32_t(g)) << a.shift) +
                                    uint32_t(p.j & ((1 << a.shift) - 1))
                              : 0u;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const uint64_t rt = uint32_t(__shfl(int(row), 16 * t + n));
      const uint64_t at = rt * (D / 2) + lg * W, st = rt * (D / kGroup4) + (lg * EPL) / kGroup4;
      gload_words<DECODE, W>(kc[t], (gptr_t)pools.kc + at);
      gload_words<DECODE, W>(vc[t], (gptr_t)pools.vc + at);
      ks[t] = pools.ks[st];
      vs[t] = pools.vs[st];
    }
  };

  constexpr int STEP = 4 * kTile4;
  int32_t x = v0 + wave * kTile4;
  At next = {};
  if (x < v1) {
    const At first = look(x);
    next = look(x + STEP);
    fetch(first);
  }
  for (; x < v1; x += STEP) {
    f32x4_t sc[4];
    const uint64_t okc = okm;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      sc[t] = zero4();
      const float ksc = scale_of(ks[t]), vsc = scale_of(vs[t]);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        Frag<bf16_t> k;
        k.v = bf16_of_codes(kc[t][kk], ksc);
        sc[t] = mma_parts<T>(k, qf[kk], sc[t]);
        *reinterpret_cast<uint4*>(vt + (16 * t + n) * RS + EPL * lg + 8 * kk) = bf16_of_codes(vc[t][kk], vsc);
      }
    }
    if (x + STEP < v1) {
      const At now = next;
      next = look(x + 2 * STEP);
      fetch(now);
    }
    float p[16];
    float mx = m;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 16 * t + 4 * lg + i;
        bool see = (okc >> key) & 1;
        if constexpr (!DECODE) {
          const int32_t j = sn.pos(x + key);
          see = see && j <= tr && (j > tr - a.W || j < a.ns);
        }
        p[4 * t + i] = see ? sc[t][i] * a.scale : -INFINITY;
        mx = fmaxf(mx, p[4 * t + i]);
      }
    mx = lg_max(mx);
    const float f = __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    l *= f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      p[i] = __builtin_amdgcn_exp2f(p[i] - m);
      l += p[i];
    }
    Parts<T> pf[2];
    pf[0].set8(p);
    pf[1].set8(p + 8);
    wave_lds_order();
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[ct][i] *= f;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
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

template <typename T, int D>
hipError_t decode_t(const PagedArgs& a, const Pools4& p, hipStream_t stream) {
  nibble_rows<T, D, NoSeqs><<<dim3(a.B * a.Hkv, a.npiece), 256, 0, stream>>>(a, p, NoSeqs());
  return hipGetLastError();
}
template <typename T, int D>
hipError_t prefill_t(const PagedArgs& a, const Pools4& p, const PagedSeqs& s, int, hipStream_t stream) {
  const dim3 grid(uint32_t(s.tile0[s.nseq]) * uint32_t(a.Hkv), a.npiece);
  nibble_rows<T, D, PagedSeqs><<<grid, 256, 0, stream>>>(a, p, s);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_nibble_decode(const PagedArgs& a, const Pools4& p, int d, int dtype, hipStream_t stream) {
  hipError_t e;
  if (dtype == GLIDE_BF16) e = d == 128 ? decode_t<bf16_t, 128>(a, p, stream) : decode_t<bf16_t, 64>(a, p, stream);
  else e = d == 128 ? decode_t<float, 128>(a, p, stream) : decode_t<float, 64>(a, p, stream);
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
