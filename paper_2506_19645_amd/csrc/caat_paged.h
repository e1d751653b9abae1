// What the kernels over a paged key / value cache share (device code).
#pragma once
#include "caat_internal.h"

namespace caat {

static constexpr int PHD = 128;                  // head dim

// Rows of sequence b: the first and how many; none unless they lie inside the packed rows.
__device__ __forceinline__ int seq_rows(const PagedArgs& a, int b, int& first) {
  if (!a.row_start) {
    first = b;
    return b < a.rows ? 1 : 0;
  }
  const int r0 = a.row_start[b], r1 = a.row_start[b + 1];
  first = r0;
  return r0 >= 0 && r1 > r0 && r1 <= a.rows ? r1 - r0 : 0;
}

__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ long long uni64(long long x) {
  return (long long)(((unsigned long long)(unsigned)uni((int)(x >> 32)) << 32) | (unsigned)uni((int)x));
}
__device__ __forceinline__ long long lane64(long long x, int lane) {   // a lane's value, `lane` uniform
  return (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32) |
                     (unsigned)__builtin_amdgcn_readlane((int)x, lane));
}

// inclusive sums over the lanes of a wave
__device__ __forceinline__ int wave_sums(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // from 1, 2, 4, 8 lanes below inside rows of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // the last lane of rows 0 and 2 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // lane 31 to rows 2 and 3
  return v;
}

// the product of two rows' eight bf16 values
__device__ __forceinline__ float dot8(const uint4& a, const uint4& b) {
  const unsigned x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
  float s = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i) s += lo_bf(x[i]) * lo_bf(y[i]) + hi_bf(x[i]) * hi_bf(y[i]);
  return s;
}

// The two forms of the attention: caat_paged_few.hip, caat_paged_prompt.hip
static constexpr int PFEW_ROWS = 32;             // the first one's share: (token, head of the group) rows of a sequence
inline bool paged_few_rows(const PagedArgs& a, int max_new) { return (long long)max_new * (a.hpr / a.kvpr) <= PFEW_ROWS; }
bool paged_few_takes(const PagedArgs& a, int max_new);
size_t paged_few_workspace_bytes(const PagedArgs& a, int max_new);
hipError_t launch_paged_few(const PagedArgs& a, int e4m3, int max_new, const bf16_t* q, bf16_t* out, const void* kc, const void* vc,
                            void* workspace, hipStream_t s);
size_t paged_prompt_workspace_bytes(const PagedArgs& a, int max_new);
hipError_t launch_paged_prompt(const PagedArgs& a, int e4m3, int max_new, const bf16_t* q, bf16_t* out, const void* kc, const void* vc,
                               void* workspace, hipStream_t s);

}  // namespace caat
