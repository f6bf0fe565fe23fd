// The 4-bit paged cache: its pools, its number format, and the launches of the
// attention over it (kernels in nibble.hip, host side in nibble_api.hip).
#pragma once

#include "paged.h"

namespace glide {

constexpr int kGroup4 = 32;  // elements of a row that share a scale

// The pools of a 4-bit cache, contiguous: codes [n_pages][Hkv][page_size][d/2],
// scales [n_pages][Hkv][page_size][d/32].
struct Pools4 {
  uint8_t *kc, *ks, *vc, *vs;
};

// Rows of a workgroup of nibble_tiles (four waves of 32, or eight).
constexpr int kRows4 = 128, kRows4Big = 256;

// a.kp, a.vp, a.kn, a.vn, a.wp and the strides are not used; as launch_paged_decode
// and launch_paged_prefill otherwise.
// tile_keys: keys of a wave's tile, 64 or (bf16) 32; tile_rows: kPagedRows
// (nibble_rows), kRows4 or kRows4Big.
hipError_t launch_nibble_decode(const PagedArgs& a, const Pools4& p, int d, int dtype, int tile_keys,
                                hipStream_t stream);
hipError_t launch_nibble_prefill(const PagedArgs& a, const Pools4& p, const PagedSeqs& s, int d, int dtype,
                                 int tile_rows, hipStream_t stream);

// Rows of a workgroup of a prefill (its first launch; pieces: of each row tile), or
// with cu_seqlens_host NULL the keys of a wave's tile of a decode; not a part of
// the library's interface (for its tests).
extern "C" int32_t glide_internal_nibble_plan(const glide_paged_config* cfg, const int32_t* cu_seqlens_host,
                                              int64_t max_len, int32_t* pieces);

// ---------------------------------------------------------------------------
// Four bits.  A value is s 2^e: s one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their
// negatives (three bits: two of exponent, one of mantissa; and a sign), e one
// byte (e + 127) for 32 elements of a row.  e is the least integer at which the
// group's largest magnitude is at most 7 * 2^e: 7 is as far from 6 (what it is
// stored as) as 5 is from its neighbours, so no element is off by more than
// 2^e, and half the groups keep a finer step than with 6 in its place.  Every
// value is a bf16 number: the matrix cores take it without another rounding.
constexpr int kMinScale = 3, kMaxScale = 252;  // e in [-124, 125]: normal numbers, and 6 * 2^125 is one
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int b = int(u >> 23) - 2 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // 7 * 2^e = 1.75 * 2^(e + 2)
  return uint32_t(b < kMinScale ? kMinScale : b > kMaxScale ? kMaxScale : b);
}
// A stored byte as a factor (bytes out of range, which no call writes, count as the nearest in it).
__device__ __forceinline__ float scale_of(uint32_t byte) {
  const uint32_t b = byte < uint32_t(kMinScale) ? kMinScale : byte > uint32_t(kMaxScale) ? kMaxScale : byte;
  return __uint_as_float(b << 23);
}
// The code of a magnitude a = |x| 2^-e, ties to the even one; *off: how far a is
// from it in its steps (1/2: a tie).  F: float or double.
template <typename F>
__device__ __forceinline__ uint32_t code_of(F a, F* off) {
  a = a < F(6) ? a : F(6);
  const uint32_t e = a < F(2) ? 0u : a < F(4) ? 1u : 2u;  // steps of 1/2, 1 and 2
  const F t = a * (e == 0 ? F(2) : e == 1 ? F(1) : F(0.5)), r = __builtin_elementwise_roundeven(t);
  *off = t < r ? r - t : t - r;
  return uint32_t(int(r)) + 2 * e;
}
// Eight values of one group to eight codes, element i in bits 4 i .. 4 i + 3.
// inv = 2^-e; *off: the largest.
__device__ __forceinline__ uint32_t codes8(const float* x, float inv, float* off) {
  uint32_t w = 0;
  float far = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float o;
    w |= (code_of(fabsf(x[i]) * inv, &o) | (x[i] < 0.f ? 8u : 0u)) << (4 * i);
    far = fmaxf(far, o);
  }
  *off = far;
  return w;
}
// Eight codes to eight bf16 values times 2^e (exact), in order.
__device__ __forceinline__ uint4 bf16_of_codes(uint32_t w, float scale) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const bf16x2_t a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
  const bf16x2_t b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
  const bf16x2_t c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
  const bf16x2_t d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
  return make_uint4(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, c),
                    __builtin_bit_cast(uint32_t, d));
}

}  // namespace glide
