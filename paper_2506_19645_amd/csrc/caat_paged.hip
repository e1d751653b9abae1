// Paged key / value cache for gfx950: the new tokens of a ragged batch are rotated and stored to the pages of their sequences,
// and attend to them.
#include <math.h>
#include <algorithm>
#include "caat_paged.h"

namespace caat {

// The sequence that owns a row (-1: none); called by whole waves, the answer is uniform.  Among many sequences the last one whose
// rows begin at or before the row is found 64 at a time; if the list does not run upwards, and so that one does not own the row,
// they are gone through.
__device__ __forceinline__ int seq_of_row(const PagedArgs& a, int row, int& first, int& n) {
  const int lane = threadIdx.x & 63;
  if (!a.row_start) {
    first = row;
    n = 1;
    return row < a.batch ? row : -1;
  }
  if (a.batch > 64) {
    int lo = 0, size = a.batch;                  // among lo .. lo + size - 1
    while (size > 1) {
      const int step = (size + 63) / 64, at = lane * step;
      const bool before = at < size && a.row_start[lo + at] <= row;
      const int k = __popcll(__ballot(before));  // (lane 0 .. k - 1, if the list runs upwards)
      if (k == 0) break;
      lo += (k - 1) * step;
      size = min(step, size - (k - 1) * step);
    }
    lo = uni(lo);
    n = seq_rows(a, lo, first);
    if (n > 0 && row >= first && row < first + n) return lo;
  }
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    int f = 0, m = 0;
    if (b0 + lane < a.batch) m = seq_rows(a, b0 + lane, f);
    const unsigned long long hit = __ballot(m > 0 && row >= f && row < f + m);
    if (hit) {
      const int l = __builtin_ctzll(hit);
      first = __shfl(f, l, 64);
      n = __shfl(m, l, 64);
      return b0 + l;
    }
  }
  return -1;
}

__device__ __forceinline__ float e4m3_clamp(float x) { return x != x ? x : fminf(fmaxf(x, -448.0f), 448.0f); }
// Quotients by s, rounded to nearest in fp32: by its significand, behind a shift by its exponent, so that any s does.  What the
// product with the rounded reciprocal lacks is exact in fp32, and its share goes to it with one rounding (Markstein, 1990); the product
// alone moves values off the middle of two codes.  Beyond the codes' range only that they are beyond.  (us, the product / this, kernel
// alone: 7047 rows of 32 heads 55.6 / 53.6, 512 rows 7.3 / 7.9, 127 rows of 64 / 8 heads 5.6 / 6.0; calls with the compiler's division
// 7047 rows 72 and not 55, 512 rows 9.8 and not 7.9.)
struct Divisor {
  float m, r;
  int e;
  __device__ __forceinline__ explicit Divisor(float s) : m(__builtin_amdgcn_frexp_mantf(s)), e(-__builtin_amdgcn_frexp_expf(s)) { r = 1.0f / m; }
  __device__ __forceinline__ float quotient(float x) const {
    x = ldexpf(x, e);
    const float q = __builtin_amdgcn_fmed3f(x * r, -480.0f, 480.0f);   // (an infinite one would leave infinity less infinity)
    return __builtin_fmaf(__builtin_fmaf(-q, m, x), r, q);
  }
};
// eight values to eight e4m3 codes
__device__ __forceinline__ uint2 pack_e4m3(const float* v) {
  uint2 w;
  int lo = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(v[0]), e4m3_clamp(v[1]), 0, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(v[2]), e4m3_clamp(v[3]), lo, true);
  int hi = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(v[4]), e4m3_clamp(v[5]), 0, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(e4m3_clamp(v[6]), e4m3_clamp(v[7]), hi, true);
  w.x = (unsigned)lo;
  w.y = (unsigned)hi;
  return w;
}

// ---------------------------------------------------------------------------------------------------------
// Append.  A workgroup owns a row on all ranks (or, of few rows, every gridDim.y-th part of its heads): the row's 64 sines and
// cosines are made once, then a thread turns 8 pairs (j, j + 64) of one q or k head at a time and moves the matching channels
// of v along with k.
template <bool STREAM> __device__ __forceinline__ uint4 take(const bf16_t* p) {
  if constexpr (STREAM) return ld_stream(p);
  return *reinterpret_cast<const uint4*>(p);
}
template <bool STREAM> __device__ __forceinline__ void put(bf16_t* p, const uint4& v) {
  if constexpr (STREAM) st_stream(p, v);
  else *reinterpret_cast<uint4*>(p) = v;
}
struct RopeTable {
  float2 rev[64];   // revolutions per position: base^(-2j/128) / (2 pi), from 64 bits, in two floats
};

// STREAM: rows and pages that no cache keeps until they are asked for again are moved with the non-temporal hint (7047 rows of 32 heads,
// 346 MB: 71.3 -> 66.8 us, 5.2 TB/s; 8192 of 32 / 8 heads on one rank, 168 MB: 40.5 -> 36.1; but 512 rows, whose 25 MB the product in
// front of the call leaves in the caches, 7.8 -> 8.8).
template <bool E4M3, bool STREAM>
__global__ __launch_bounds__(256) void paged_append_kernel(const PagedArgs a, const RopeTable rt, const bf16_t* qkv, bf16_t* q_out,
                                                           long long ld_qkv, void* kc, void* vc) {
  __shared__ float s_cs[64], s_sn[64];
  const int row = blockIdx.x, tid = threadIdx.x;
  int first, n;
  const int b = seq_of_row(a, row, first, n);
  if (b < 0) return;
  const int pos = max(a.lens[b], 0) - n + (row - first);
  if (tid < 64) {
    float sn, cs;
    rope_sincos((float)pos, rt.rev[tid], sn, cs);
    s_cs[tid] = cs;
    s_sn[tid] = sn;
  }
  __syncthreads();
  const int col = pos / a.page_size;
  const int page = pos >= 0 && col < a.max_pages ? a.table[(long long)b * a.max_pages + col] : -1;
  const bool store = page >= 0 && page < a.n_pages;
  const long long slot = (long long)page * a.s_page + (long long)(pos - col * a.page_size) * a.s_row;
  const int per = (a.hpr + a.kvpr) * 8;
  for (int u = blockIdx.y * 256 + tid; u < a.T * per; u += gridDim.y * 256) {
    const int rank = u / per, rem = u - rank * per;
    const int head = rem >> 3, grp = rem & 7;
    const bf16_t* src = qkv + ((long long)rank * a.rows + row) * ld_qkv + head * PHD + grp * 8;
    const bool is_k = head >= a.hpr;
    float ks = 1.0f, vs = 1.0f;
    if constexpr (E4M3) {                        // on their way with the row's values (7047 rows of 32 heads 57.9 -> 53.6 us)
      if (is_k && a.k_scale) ks = a.k_scale[rank * a.kvpr + head - a.hpr];
      if (is_k && a.v_scale) vs = a.v_scale[rank * a.kvpr + head - a.hpr];
    }
    const uint4 lo = take<STREAM>(src), hi = take<STREAM>(src + 64);
    const unsigned lw[4] = {lo.x, lo.y, lo.z, lo.w}, hw[4] = {hi.x, hi.y, hi.z, hi.w};
    float y1[8], y2[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x1 = e & 1 ? hi_bf(lw[e >> 1]) : lo_bf(lw[e >> 1]), x2 = e & 1 ? hi_bf(hw[e >> 1]) : lo_bf(hw[e >> 1]);
      const float cs = s_cs[grp * 8 + e], sn = s_sn[grp * 8 + e];
      y1[e] = x1 * cs - x2 * sn;
      y2[e] = x2 * cs + x1 * sn;
    }
    if (!is_k || !E4M3) {
      const uint4 r1 = make_uint4(pack2bf(y1[0], y1[1]), pack2bf(y1[2], y1[3]), pack2bf(y1[4], y1[5]), pack2bf(y1[6], y1[7]));
      const uint4 r2 = make_uint4(pack2bf(y2[0], y2[1]), pack2bf(y2[2], y2[3]), pack2bf(y2[4], y2[5]), pack2bf(y2[6], y2[7]));
      bf16_t* dst = is_k ? (bf16_t*)kc + rank * a.s_rank + slot + (head - a.hpr) * a.s_head + grp * 8
                         : q_out + ((long long)rank * a.rows + row) * a.ld_q + head * PHD + grp * 8;
      if (!is_k || store) {
        put<STREAM>(dst, r1);
        put<STREAM>(dst + 64, r2);
      }
    }
    if (is_k && store) {
      const int kvh = head - a.hpr;
      const uint4 vlo = take<STREAM>(src + a.kvpr * PHD), vhi = take<STREAM>(src + a.kvpr * PHD + 64);
      const long long at = rank * a.s_rank + slot + kvh * a.s_head + grp * 8;
      if constexpr (E4M3) {
        unsigned char *k8 = (unsigned char*)kc + at, *v8 = (unsigned char*)vc + at;
        const Divisor by_ks(ks), by_vs(vs);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          y1[e] = by_ks.quotient(y1[e]);
          y2[e] = by_ks.quotient(y2[e]);
        }
        *reinterpret_cast<uint2*>(k8) = pack_e4m3(y1);
        *reinterpret_cast<uint2*>(k8 + 64) = pack_e4m3(y2);
        const unsigned vw[8] = {vlo.x, vlo.y, vlo.z, vlo.w, vhi.x, vhi.y, vhi.z, vhi.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          y1[2 * e] = by_vs.quotient(lo_bf(vw[e]));
          y1[2 * e + 1] = by_vs.quotient(hi_bf(vw[e]));
          y2[2 * e] = by_vs.quotient(lo_bf(vw[4 + e]));
          y2[2 * e + 1] = by_vs.quotient(hi_bf(vw[4 + e]));
        }
        *reinterpret_cast<uint2*>(v8) = pack_e4m3(y1);
        *reinterpret_cast<uint2*>(v8 + 64) = pack_e4m3(y2);
      } else {
        put<STREAM>((bf16_t*)vc + at, vlo);
        put<STREAM>((bf16_t*)vc + at + 64, vhi);
      }
    }
  }
}

hipError_t launch_paged_append(const PagedArgs& a, int e4m3, const bf16_t* qkv, bf16_t* q_out, long long ld_qkv, void* kc, void* vc,
                               float rope_base, hipStream_t s) {
  if (a.rows == 0) return hipSuccess;
  RopeTable rt;
  const double step = exp2(-2.0 / PHD * log2((double)rope_base));
  double rev = 1.0 / 6.283185307179586476925;
  for (int j = 0; j < 64; ++j, rev *= step) {    // 63 roundings to 53 bits
    rt.rev[j].x = (float)rev;
    rt.rev[j].y = (float)(rev - (double)rt.rev[j].x);
  }
  const int units = a.T * (a.hpr + a.kvpr) * 8;
  // (8 ranks of 4 + 4 + 4 heads: 400 rows 8.8 us whole, 8.2 in two parts, 600 rows 10.8 and 9.7, 1500 rows 24.2 and 25.4)
  const int parts = a.rows < 1024 ? (units + 255) / 256 : 1;
  const dim3 grid((unsigned)a.rows, (unsigned)parts);
  // rows read, q and the pages' rows written: more than 96 MB of them is taken to be too much for the caches
  const bool stream = (long long)a.T * a.rows * PHD * (4 * a.hpr + (e4m3 ? 6 : 8) * a.kvpr) > (96LL << 20);
  auto kernel = e4m3 ? (stream ? paged_append_kernel<true, true> : paged_append_kernel<true, false>)
                     : (stream ? paged_append_kernel<false, true> : paged_append_kernel<false, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a, rt, qkv, q_out, ld_qkv, kc, vc);
  return hipGetLastError();
}

// The most that calls with as many new tokens or fewer take, whatever their rows, sequences and tables: a program sizes it once.
size_t paged_attn_workspace_bytes(const PagedArgs& a, int max_new) {
  const int few = std::min(max_new, PFEW_ROWS / (a.hpr / a.kvpr));   // the most that the few tokens' kernel is given
  const size_t bytes = paged_prompt_workspace_bytes(a, max_new);
  return few > 0 ? std::max(bytes, paged_few_workspace_bytes(a, few)) : bytes;
}

hipError_t launch_paged_attn(const PagedArgs& a, int e4m3, const bf16_t* q, bf16_t* out, const void* kc, const void* vc, int max_new,
                             void* workspace, hipStream_t s) {
  if (paged_few_takes(a, max_new)) return launch_paged_few(a, e4m3, max_new, q, out, kc, vc, workspace, s);
  return launch_paged_prompt(a, e4m3, max_new, q, out, kc, vc, workspace, s);
}

}  // namespace caat
