// Launch descriptors of the calls that fill a paged cache (kernels in
// append.hip): new rows with the position rotation, into a cache of the call's
// element type or of 4 bits; page bounds; rows of a 4-bit cache read back.
#pragma once

#include "nibble.h"

namespace glide {

// Tokens of one workgroup of append_rotated, at most, where it does not keep
// page bounds (with them a workgroup has a page's tokens).
constexpr int kAppendTokens = 64;

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
// Of the pages with new tokens; seqs.tile0: pages of each sequence, as launch_append with unit = shift.
hipError_t launch_new_bounds(const AppendArgs& a, const PagedSeqs& s, int d, int dtype, hipStream_t stream);
hipError_t launch_read4(const AppendArgs& a, const PagedSeqs& s, char* ko, char* vo, int d, int dtype,
                        hipStream_t stream);

}  // namespace glide
