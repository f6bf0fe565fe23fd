// Launch descriptors of the calls that fill a paged cache (kernels in
// append.hip): new rows with the position rotation, into a cache of the call's
// element type or of 4 bits; page bounds; rows of a 4-bit cache read back.
#pragma once

#include "paged.h"

namespace glide {

constexpr int kGroup4 = 32;  // elements of a row that share a scale in a 4-bit cache
// Tokens of one workgroup of append_rotated, where no page bounds are kept
// (with them a workgroup has a page's tokens).
constexpr int kAppendTokens = 64;

// The pools of a 4-bit cache, contiguous: codes [n_pages][Hkv][page_size][d/2],
// scales [n_pages][Hkv][page_size][d/32].
struct Pools4 {
  uint8_t *kc, *ks, *vc, *vs;
};

struct AppendArgs {
  const char *q, *k, *v;  // q: NULL where none is to be rotated
  char* qo;
  const float* freqs;     // radians per position and pair; rot = 0: not read
  const int32_t* pos;     // positions of the new tokens; NULL: theirs in the cache
  char *kp, *vp;          // pools of the call's type, with strides in bytes
  float* wp;
  int64_t ks[3], vs[3];
  Pools4 p4;
  char* bounds;           // [n_pages][Hkv][2][d], or NULL
  const int32_t *table, *lens;
  int32_t B, Hq, Hkv, G;
  int32_t n_pages, max_pages, shift, cap;
  int32_t rot;            // leading elements of a row that are rotated
  int32_t unit;           // log2 of the tokens of a workgroup, which start at a multiple of them
};

// seqs.tile0: workgroups (per KV head) of each sequence
hipError_t launch_append(const AppendArgs& a, const PagedSeqs& s, int d, int dtype, bool four, bool interleaved,
                         hipStream_t stream);
// keys: tokens of a sequence, at most (it sizes a grid only)
hipError_t launch_page_bounds(const AppendArgs& a, int64_t keys, int d, int dtype, hipStream_t stream);
hipError_t launch_read4(const AppendArgs& a, const PagedSeqs& s, char* ko, char* vo, int d, int dtype,
                        hipStream_t stream);

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
// Eight values of one group to eight codes, element i in bits 4 i .. 4 i + 3;
// ties to the even code.  inv = 2^-e.
__device__ __forceinline__ uint32_t codes8(const float* x, float inv) {
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = fminf(fabsf(x[i]) * inv, 6.f);
    const uint32_t e = a < 2.f ? 0u : a < 4.f ? 1u : 2u;  // steps of 1/2, 1 and 2
    const float r = __builtin_rintf(a * (e == 0 ? 2.f : e == 1 ? 1.f : 0.5f));
    const uint32_t c = uint32_t(int(r)) + 2 * e;
    w |= (c | (x[i] < 0.f ? 8u : 0u)) << (4 * i);
  }
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
