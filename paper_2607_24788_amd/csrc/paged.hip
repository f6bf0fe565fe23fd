// Softmax attention over a paged key-value cache: sliding window, sinks,
// grouped query heads, pieces of long rows joined, attention weights.
#include <algorithm>

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
// New rows into their pages: one 16-byte piece of K and of V per thread; the
// weights of new tokens start from 0.  Copies; bound by launch and memory.
template <int ROW>  // bytes of a row
__global__ __launch_bounds__(256) void paged_append(PagedArgs a, PagedSeqs s, const char* k, const char* v) {
  constexpr int P = ROW / 16;
  const int i = blockIdx.y;  // sequence of the launch
  const int b = s.seq0 + i;
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  const int64_t n = int64_t(s.len[i]) * a.Hkv * P;
  if (x >= n) return;
  const int c = int(x % P);
  const int64_t row = x / P;  // token, head
  const int g = int(row % a.Hkv);
  const int32_t j = seq_len(a, b) - s.len[i] + int32_t(row / a.Hkv);
  if (j < 0) return;
  const Slot sl = paged_slot(a.table + int64_t(b) * a.max_pages, j, a.shift, a.n_pages);
  if (!sl.ok) return;
  const int64_t src = (int64_t(s.start[i]) * a.Hkv + row) * ROW + c * 16;
  *reinterpret_cast<uint4*>(a.kp + slot_offset(a.ks, sl, g) + c * 16) = *reinterpret_cast<const uint4*>(k + src);
  *reinterpret_cast<uint4*>(a.vp + slot_offset(a.vs, sl, g) + c * 16) = *reinterpret_cast<const uint4*>(v + src);
}

__global__ __launch_bounds__(256) void paged_clear_weights(PagedArgs a, PagedSeqs s) {
  const int i = blockIdx.y, b = s.seq0 + i;
  const int64_t x = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (x >= int64_t(s.len[i]) * a.Hkv) return;
  const int g = int(x % a.Hkv);
  const int32_t j = seq_len(a, b) - s.len[i] + int32_t(x / a.Hkv);
  if (j < 0) return;
  const Slot sl = paged_slot(a.table + int64_t(b) * a.max_pages, j, a.shift, a.n_pages);
  if (sl.ok) a.wp[((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot] = 0.f;
}

// ---------------------------------------------------------------------------
// Attention of one tile of 16 rows ((token, head) pairs of one KV head) over
// one piece of the tokens that they see; the four waves take tiles of 32 keys
// in turn, each with a running maximum and sum of its own, joined at the end.
//   S^T = K Q^T (keys are the MFMA rows): a lane holds 8 scores of one row,
//   already the right operand of O^T += V^T P^T with keys in the order
//   4g + 0..3, 16 + 4g + 0..3; V goes through LDS for its columns.
template <typename T, int D, bool DECODE>
__global__ __launch_bounds__(256) void attend_rows(PagedArgs a, PagedSeqs s) {
  constexpr int KK = D / 32, CT = D / 16, RS = D + 16 / int(sizeof(T)), ES = int(sizeof(T));
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
  const int32_t len = seq_len(a, b);
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
  const int32_t v0 = int32_t(blockIdx.y) * pl, v1 = v0 + pl < sn.n ? v0 + pl : sn.n;
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  const char* zr = reinterpret_cast<const char*>(zero_row);

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

  if constexpr (DECODE) {
    // the new token's rows into their page
    if (a.kn && blockIdx.y == 0 && len > 0 && threadIdx.x < 2 * D * ES / 16) {
      const Slot sl = paged_slot(trow, len - 1, a.shift, a.n_pages);
      const int c = (threadIdx.x % (D * ES / 16)) * 16;
      const bool val = threadIdx.x >= D * ES / 16;
      const uint4 x = *reinterpret_cast<const uint4*>((val ? a.vn : a.kn) + (int64_t(b) * a.Hkv + g) * D * ES + c);
      if (sl.ok)
        *reinterpret_cast<uint4*>((val ? a.vp + slot_offset(a.vs, sl, g) : a.kp + slot_offset(a.ks, sl, g)) + c) = x;
    }
  }

  for (int32_t x = v0 + wave * kPagedTile; x < v1; x += 4 * kPagedTile) {
    Frag<T> kf[2][KK], vf[2][KK];
    uint32_t ok[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int32_t vi = x + 16 * t + n;
      bool good = vi < v1;
      const int32_t j = good ? sn.pos(vi) : 0;
      Slot sl = {0, 0, false};
      if (good) sl = paged_slot(trow, j, a.shift, a.n_pages);
      good = good && sl.ok;
      const char* kr = good ? a.kp + slot_offset(a.ks, sl, g) : zr;
      const char* vr = good ? a.vp + slot_offset(a.vs, sl, g) : zr;
      if constexpr (DECODE) {
        if (a.kn && good && j == len - 1) {
          kr = a.kn + (int64_t(b) * a.Hkv + g) * D * ES;
          vr = a.vn + (int64_t(b) * a.Hkv + g) * D * ES;
        }
      }
      ok[t] = uint32_t(__ballot(good)) & 0xffffu;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        kf[t][kk].load(reinterpret_cast<const T*>(kr) + 32 * kk + 8 * lg);
        vf[t][kk].load(reinterpret_cast<const T*>(vr) + 32 * kk + 8 * lg);
      }
    }
    f32x4_t sc[2] = {zero4(), zero4()};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) {
        sc[t] = mma(kf[t][kk], qf[kk], sc[t]);
        T* w = vt + (16 * t + n) * RS + 32 * kk + 8 * lg;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<uint4*>(w) = vf[t][kk].v;
        } else {
          reinterpret_cast<float4*>(w)[0] = make_float4(vf[t][kk].v[0], vf[t][kk].v[1], vf[t][kk].v[2], vf[t][kk].v[3]);
          reinterpret_cast<float4*>(w)[1] = make_float4(vf[t][kk].v[4], vf[t][kk].v[5], vf[t][kk].v[6], vf[t][kk].v[7]);
        }
      }
    float p[8];
    float mx = m;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = 4 * lg + i;
        bool see = (ok[t] >> key) & 1;
        if constexpr (!DECODE) {
          const int32_t j = sn.pos(x + 16 * t + key);
          see = see && j <= tr && (j > tr - a.W || j < a.ns);
        }
        p[4 * t + i] = see ? sc[t][i] * a.scale : -INFINITY;
        mx = fmaxf(mx, p[4 * t + i]);
      }
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
    pf.set8(p);  // bf16: weights rounded to half a step, 2^-9 of each
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
  const bool split = a.npiece > 1;
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

// The pieces of a row joined: a wave per row, D / 64 elements per lane.
template <typename T, int D>
__global__ __launch_bounds__(256) void paged_join(PagedArgs a, int64_t row0, int64_t rows) {
  const int lane = threadIdx.x & 63;
  const int64_t r = row0 + int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6);
  if (r >= row0 + rows) return;
  const float* ml = a.ml + r * a.npiece * 2;
  float M = kNoMax;
  for (int i = 0; i < a.npiece; ++i) M = fmaxf(M, ml[2 * i]);
  float L = 0.f, x[D / 64] = {};
  for (int i = 0; i < a.npiece; ++i) {
    const float li = ml[2 * i + 1];
    if (li == 0.f) continue;  // no key of this piece has a part in the row
    const float f = __builtin_amdgcn_exp2f(ml[2 * i] - M);
    L += li * f;
#pragma unroll
    for (int e = 0; e < D / 64; ++e) x[e] += f * a.acc[(r * a.npiece + i) * D + lane * (D / 64) + e];
  }
  const float inv = L == 0.f ? 0.f : 1.f / L;
#pragma unroll
  for (int e = 0; e < D / 64; ++e)
    reinterpret_cast<T*>(a.out)[r * D + lane * (D / 64) + e] = from_f32<T>(x[e] * inv);
  if (lane == 0) {
    const float lse2 = L > 0.f ? M + __builtin_amdgcn_logf(L) : L == 0.f ? -INFINITY : L;
    if (a.lse) a.lse[r] = lse2 * kLn2;
    if (a.lse2) a.lse2[r] = lse2;
  }
}

// ---------------------------------------------------------------------------
// Decode: weights_j += sum over the group's heads of e^{s_j - lse}, from the
// raw scores that the attention left.  One thread per visible token.
__global__ __launch_bounds__(256) void decode_weights(PagedArgs a) {
  const int b = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv;
  const int32_t len = seq_len(a, b);
  if (len == 0) return;
  const Seen sn = seen_by(len - 1, len - 1, a.W, a.ns);
  const int32_t v0 = blockIdx.y * 256 + threadIdx.x;
  // the appended token's weight starts from 0, also where it is not seen
  const bool fresh = a.kn && v0 == 0 && (sn.n == 0 || sn.pos(sn.n - 1) != len - 1);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  if (fresh) {
    const Slot sl = paged_slot(trow, len - 1, a.shift, a.n_pages);
    if (sl.ok) a.wp[((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot] = 0.f;
  }
  for (int32_t v = v0; v < sn.n; v += int32_t(gridDim.y) * 256) {
    const int32_t j = sn.pos(v);
    const Slot sl = paged_slot(trow, j, a.shift, a.n_pages);
    if (!sl.ok) continue;
    float w = 0.f;
    for (int h = 0; h < a.G; ++h) {
      const int64_t r = int64_t(b) * a.Hq + g * a.G + h;
      const float z = a.lse2[r];
      w += z == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(a.scores[r * a.nv + v] - z);
    }
    float* at = a.wp + ((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot;
    *at = (a.kn && j == len - 1 ? 0.f : *at) + w;
  }
}

// Prefill: the last n_observe queries of each sequence.  A wave owns 32 keys
// (in registers) and goes through the scored rows in order: no sum's order
// depends on timing.
template <typename T, int D>
__global__ __launch_bounds__(256) void prefill_weights(PagedArgs a, PagedSeqs s, int n_observe) {
  constexpr int KK = D / 32;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, lg = lane >> 4;
  const int i = blockIdx.x / a.Hkv, g = blockIdx.x % a.Hkv, b = s.seq0 + i;
  const int32_t len = seq_len(a, b), ntok = s.len[i], p0 = len - ntok;
  const int32_t obs = ntok < n_observe ? ntok : n_observe;
  if (len == 0 || obs == 0) return;
  const int32_t first = ntok - obs;  // first scored token
  const int32_t t0 = p0 + first > 0 ? p0 + first : 0;
  const Seen sn = seen_by(t0, len - 1, a.W, a.ns);
  const int32_t* trow = a.table + int64_t(b) * a.max_pages;
  for (int32_t x = blockIdx.y * 128 + wave * 32; x < sn.n; x += int32_t(gridDim.y) * 128) {
    Frag<T> kf[2][KK];
    uint32_t ok[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int32_t vi = x + 16 * t + n;
      Slot sl = {0, 0, false};
      if (vi < sn.n) sl = paged_slot(trow, sn.pos(vi), a.shift, a.n_pages);
      ok[t] = uint32_t(__ballot(sl.ok)) & 0xffffu;
      const char* kr = sl.ok ? a.kp + slot_offset(a.ks, sl, g) : reinterpret_cast<const char*>(zero_row);
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[t][kk].load(reinterpret_cast<const T*>(kr) + 32 * kk + 8 * lg);
    }
    float w[2][4] = {};
    const int32_t rend = ntok * a.G;
    for (int32_t rb = first * a.G; rb < rend; rb += 16) {
      const bool rok = rb + n < rend;
      const int32_t r = rok ? rb + n : rend - 1, tr = rok ? p0 + r / a.G : -1;
      const int64_t orow = (int64_t(s.start[i]) + r / a.G) * a.Hq + g * a.G + r % a.G;
      const float z = a.lse2[orow];
      Frag<T> qf[KK];
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) qf[kk].load(reinterpret_cast<const T*>(a.q) + orow * D + 32 * kk + 8 * lg);
      f32x4_t sc[2] = {zero4(), zero4()};
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) sc[t] = mma(kf[t][kk], qf[kk], sc[t]);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int key = 4 * lg + e;
          const int32_t j = sn.pos(x + 16 * t + key);
          const bool see = ((ok[t] >> key) & 1) && j <= tr && (j > tr - a.W || j < a.ns) && z != -INFINITY;
          w[t][e] += see ? __builtin_amdgcn_exp2f(sc[t][e] * a.scale - z) : 0.f;
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float y = dpp_sum_rows<16>(w[t][e]);
        const int key = 4 * lg + e;
        const int32_t vi = x + 16 * t + key;
        if (n == 0 && vi < sn.n && ((ok[t] >> key) & 1)) {
          const Slot sl = paged_slot(trow, sn.pos(vi), a.shift, a.n_pages);
          a.wp[((int64_t(sl.page) * a.Hkv + g) << a.shift) + sl.slot] += y;
        }
      }
  }
}

template <typename T, int D>
hipError_t attend_t(const PagedArgs& a, const PagedSeqs* s, hipStream_t stream) {
  static const PagedSeqs none = {};
  if (!s) {
    attend_rows<T, D, true><<<dim3(a.B * a.Hkv, a.npiece), 256, 0, stream>>>(a, none);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.npiece == 1) return e;
    const int64_t rows = int64_t(a.B) * a.Hq;
    paged_join<T, D><<<dim3(uint32_t((rows + 3) / 4)), 256, 0, stream>>>(a, 0, rows);
    return hipGetLastError();
  }
  const int64_t tiles = s->tile0[s->nseq];
  if (tiles == 0) return hipSuccess;
  attend_rows<T, D, false><<<dim3(uint32_t(tiles * a.Hkv), a.npiece), 256, 0, stream>>>(a, *s);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.npiece == 1) return e;
  const int64_t row0 = int64_t(s->start[0]) * a.Hq;
  const int64_t rows = (int64_t(s->start[s->nseq - 1]) + s->len[s->nseq - 1]) * a.Hq - row0;
  paged_join<T, D><<<dim3(uint32_t((rows + 3) / 4)), 256, 0, stream>>>(a, row0, rows);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append(const PagedArgs& a, const PagedSeqs& s, const void* k, const void* v, int d, int dtype,
                               hipStream_t stream) {
  int32_t most = 0;
  for (int i = 0; i < s.nseq; ++i) most = s.len[i] > most ? s.len[i] : most;
  if (most == 0) return hipSuccess;
  const int row = d * (dtype == GLIDE_BF16 ? 2 : 4);
  if (k) {
    const int64_t n = int64_t(most) * a.Hkv * (row / 16);
    const dim3 grid(uint32_t((n + 255) / 256), s.nseq);
    const char *kc = static_cast<const char*>(k), *vc = static_cast<const char*>(v);
    if (row == 128) paged_append<128><<<grid, 256, 0, stream>>>(a, s, kc, vc);
    else if (row == 256) paged_append<256><<<grid, 256, 0, stream>>>(a, s, kc, vc);
    else paged_append<512><<<grid, 256, 0, stream>>>(a, s, kc, vc);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (k && a.wp) {
    paged_clear_weights<<<dim3(uint32_t((int64_t(most) * a.Hkv + 255) / 256), s.nseq), 256, 0, stream>>>(a, s);
    return hipGetLastError();
  }
  return hipSuccess;
}

hipError_t launch_paged_attend(const PagedArgs& a, const PagedSeqs* s, int d, int dtype, hipStream_t stream) {
  if (dtype == GLIDE_BF16) return d == 128 ? attend_t<bf16_t, 128>(a, s, stream) : attend_t<bf16_t, 64>(a, s, stream);
  return d == 128 ? attend_t<float, 128>(a, s, stream) : attend_t<float, 64>(a, s, stream);
}

hipError_t launch_paged_weights(const PagedArgs& a, const PagedSeqs* s, int n_observe, int64_t keys, int d, int dtype,
                                hipStream_t stream) {
  if (!s) {
    decode_weights<<<dim3(a.B * a.Hkv, uint32_t(std::min<int64_t>((keys + 255) / 256, 4096))), 256, 0, stream>>>(a);
    return hipGetLastError();
  }
  const dim3 grid(s->nseq * a.Hkv, uint32_t(std::min<int64_t>((keys + 127) / 128, 4096)));
  if (dtype == GLIDE_BF16) {
    if (d == 128) prefill_weights<bf16_t, 128><<<grid, 256, 0, stream>>>(a, *s, n_observe);
    else prefill_weights<bf16_t, 64><<<grid, 256, 0, stream>>>(a, *s, n_observe);
  } else {
    if (d == 128) prefill_weights<float, 128><<<grid, 256, 0, stream>>>(a, *s, n_observe);
    else prefill_weights<float, 64><<<grid, 256, 0, stream>>>(a, *s, n_observe);
  }
  return hipGetLastError();
}

}  // namespace glide
