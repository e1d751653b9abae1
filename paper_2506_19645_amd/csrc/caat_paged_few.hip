// Attention of few new tokens per sequence (decode steps, drafted tokens) over a paged key / value cache, gfx950.
//
// What bounds it: the K / V rows, read once from HBM.  The unit of work is a tile of 16 (token, query head of the group) rows of
// one sequence, rank and key / value head, times a block of keys (16 in bf16, 32 in e4m3: 8 KB of K and V).  The blocks of
// all units stand in one line, sequence by sequence, and every WAVE of the launch takes an equal stretch of it, so a batch of
// one long and many short sequences fills the chip like an even one, whatever the lengths (which only the device
// knows).  A wave copies its blocks global -> LDS into two slots that only it reads, waits for its own copies alone, and computes
// S = K q^T and O^T += V^T P with MFMAs (columns = query rows; most are idle for multi-head attention, but the matrix unit has
// nothing else to do).  P goes in as a sum of two bf16 values, 16 bits of it; a wave whose sums are not finite
// (infinity times the second value's zero) repeats its keys with fp32 MFMAs.  A unit inside one stretch is finished there; of
// one that crosses stretches every wave (or, inside it, every workgroup) leaves its sums, maximum and denominator in the
// workspace, and a second kernel joins them in the order of the keys.
#include <math.h>
#include <algorithm>
#include <type_traits>
#include "caat_paged.h"

namespace caat {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t* lds_s4_t;
typedef __attribute__((address_space(3))) const char* lds_c_t;

static constexpr int FNW = 4;                    // waves per workgroup, two slots each: 64 KB, two workgroups per compute unit
static constexpr int FNS = 2;
static constexpr int FNI = 8;                    // 1 KB copies per block: 4 of K, 4 of V
static constexpr int FPR = PHD + 4;              // floats of a partial row: 128 sums, maximum, denominator, 2 unused
static constexpr int FMAX_WGS = 512;             // workgroups of a launch
static constexpr long long FSLOT = 16 * FPR;     // floats of a partial result

// What the wave in which a unit begins says about it, if it ends in another one.
struct FewJoin {
  int rows;                                      // 0: nothing to join
  int rank, kvh, first, tile;
  int unused;
  long long begin, end, per;                     // blocks of the unit in the line of all blocks; length of a stretch
};

// Swizzles of the 16-byte chunks of a row in LDS (256-byte rows in bf16, 128 in e4m3): K is read 16 rows x one chunk at a
// time, V by the transpose read, 8 rows x two chunks for 32 lanes; each spread over all banks.
template <bool E4M3> __device__ __forceinline__ int fk_swz(int row) { return E4M3 ? (row >> 1) & 7 : row & 15; }
template <bool E4M3> __device__ __forceinline__ int fv_swz(int row) { return E4M3 ? ((row >> 1) & 3) << 1 : (row & 7) << 1; }

__device__ __forceinline__ unsigned fp8_lo(unsigned w) {   // codes 0, 1 of w as two bf16 (exact)
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false));
}
__device__ __forceinline__ unsigned fp8_hi(unsigned w) {
  return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true));
}

// A chunk of 64 sequences in registers: lane l holds sequence at + l
struct SeqChunk {
  int at, first, n, len;
  long long work;                                // blocks of one (rank, key / value head)
};

template <bool E4M3>
__global__ __launch_bounds__(64 * FNW) void paged_few_kernel(const PagedArgs a, const bf16_t* __restrict__ q, bf16_t* __restrict__ out,
                                                             const void* __restrict__ kc, const void* __restrict__ vc,
                                                             float* __restrict__ part, FewJoin* __restrict__ joins, float scale_log2,
                                                             int least, int whole) {
  constexpr int KB = E4M3 ? 32 : 16;             // keys per block
  constexpr int HV = KB / 16;                    // groups of 16 keys, each inside one page
  constexpr int ELT = E4M3 ? 1 : 2;
  constexpr int RPC = 1024 / (PHD * ELT);        // rows per copy: 4 or 8
  constexpr int CPR = 64 / RPC;                  // 16-byte chunks per row
  __shared__ uint4 ring[FNW * FNS * FNI * 64];
  static_assert(FNW * 16 * FPR * 4 <= FNW * FNS * FNI * 1024, "the partial results take the rings' place");
  __shared__ float s_m[FNW][16], s_l[FNW][16];
  const int lane = threadIdx.x & 63;
  const int wave = uni(threadIdx.x >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int grp = a.hpr / a.kvpr, heads = a.T * a.kvpr;
  const int wid = blockIdx.x * FNW + wave;
  const long long cap = (long long)a.max_pages * a.page_size;

  // ---- the line of all blocks, and this wave's stretch of it
  auto load_seqs = [&](int at) {
    SeqChunk c;
    c.at = at;
    c.first = c.n = c.len = 0;
    c.work = 0;
    if (at + lane < a.batch) {
      c.n = seq_rows(a, at + lane, c.first);
      c.len = max(a.lens[at + lane], 0);
      const long long keys = min((long long)c.len, cap);
      const long long nb = whole ? 1 : max((keys + KB - 1) / KB, 1LL);
      c.work = ((long long)c.n * grp + 15) / 16 * nb;
    }
    return c;
  };
  SeqChunk sq = load_seqs(0);
  long long total = sq.work;
  for (int at = 64; at < a.batch; at += 64) total += load_seqs(at).work;
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) total += __shfl_xor(total, off, 64);
  total = uni64(total) * heads;
  const int nwaves = gridDim.x * FNW;
  const long long per = max((total + nwaves - 1) / nwaves, (long long)least);
  const long long x0 = wid * per, x1 = min(x0 + per, total);
  FewJoin join = {};
  if (x0 < x1) {
    // the sequence of block x0: `base` is the place of its first block
    int b = 0;
    long long base = 0;
    for (;;) {
      long long incl = sq.work;
#pragma unroll
      for (int off = 1; off < 64; off <<= 1) {
        const long long up = __shfl_up(incl, off, 64);
        if (lane >= off) incl += up;
      }
      const unsigned long long over = __ballot(base + incl * heads > x0);
      if (over) {
        b = __builtin_ctzll(over);
        base += lane64(incl - sq.work, b) * heads;
        b += sq.at;
        break;
      }
      base += lane64(incl, 63) * heads;          // (some chunk holds x0 < total)
      sq = load_seqs(sq.at + 64);
    }
    int pages = -1, page0 = -1, pages_of = -1;   // lane l: entry page0 + l of sequence pages_of's table, -1: no page
    uint4* mine = ring + wave * (FNS * FNI * 64);

    for (long long x = x0; x < x1;) {
      const int sl = b - sq.at;
      const int n = __builtin_amdgcn_readlane(sq.n, sl), first = __builtin_amdgcn_readlane(sq.first, sl);
      const int len = __builtin_amdgcn_readlane(sq.len, sl);
      const long long work = lane64(sq.work, sl);
      const int keys = (int)min((long long)len, cap);
      const int nblk = (keys + KB - 1) / KB;     // may be 0
      const int nb = whole ? 1 : max(nblk, 1);
      const int tiles = (n * grp + 15) >> 4;
      const long long o = x - base;
      const long long u = (o >> 32) ? o / nb : (long long)((unsigned)o / (unsigned)nb);
      const int from = (int)(o - u * nb);
      const int to = (int)min((long long)nb, from + (x1 - x));
      const int h = (int)(u / tiles), tile = (int)(u - (long long)h * tiles);
      const int rank = h / a.kvpr, kvh = h - rank * a.kvpr;
      const int k0 = whole ? 0 : from, k1 = whole ? nblk : min(to, nblk);   // blocks of keys

      // ---- pages: the table's entries from the first one on
      auto take_pages = [&](int col) {
        page0 = col;
        pages_of = b;
        pages = -1;
        if (col + lane < a.max_pages) pages = a.table[(long long)b * a.max_pages + col + lane];
        if (pages >= a.n_pages) pages = -1;
        asm volatile("" : "+v"(pages));          // the wait for the load stands here and not in the loop over the blocks
      };
      int col = k0 * KB / a.page_size;           // of the next 16 keys to copy
      int inpage = k0 * KB - col * a.page_size;
      if (pages_of != b || col < page0 || col >= page0 + 64) take_pages(col);

      // ---- copies of a block; they return which of its groups of 16 keys have a page
      const unsigned char* kh = (const unsigned char*)kc + (rank * a.s_rank + kvh * a.s_head) * ELT;
      const unsigned char* vh = (const unsigned char*)vc + (rank * a.s_rank + kvh * a.s_head) * ELT;
      const unsigned row_bytes = (unsigned)(a.s_row * ELT);
      unsigned ko[4 / HV], vo[4 / HV];           // memory-side offsets of a group's copies
#pragma unroll
      for (int i = 0; i < 4 / HV; ++i) {
        const int row = i * RPC + lane / CPR, ch = lane % CPR;
        ko[i] = row * row_bytes + ((ch ^ fk_swz<E4M3>(row)) << 4);
        vo[i] = row * row_bytes + ((ch ^ fv_swz<E4M3>(row)) << 4);
      }
      auto copy = [&](int blk, int slot) {
        unsigned have = 0;
#pragma unroll
        for (int hv = 0; hv < HV; ++hv) {
          const int left = blk < k1 ? keys - blk * KB - hv * 16 : 0;   // keys from this group on
          int page = -1;
          if (left > 0) {
            if (col >= page0 + 64) take_pages(col);
            page = __builtin_amdgcn_readlane(pages, col - page0);
          }
          const long long at = page < 0 ? 0 : (page * a.s_page + inpage * a.s_row) * ELT;
          const i32x4_t rk = make_rsrc(kh + at), rv = make_rsrc(vh + at);
          const int rows = page < 0 ? 0 : left;
          uint4* dk = mine + slot * (FNI * 64) + hv * (4 / HV) * 64;
          uint4* dv = dk + 4 * 64;
#pragma unroll
          for (int i = 0; i < 4 / HV; ++i) {
            const bool ok = i * RPC + lane / CPR < rows;
            dma16<true>(rk, ok ? ko[i] : 0x80000000u, dk + i * 64);
            dma16<true>(rv, ok ? vo[i] : 0x80000000u, dv + i * 64);
          }
          if (page >= 0) have |= 1u << hv;
          inpage += 16;
          if (inpage >= a.page_size) {
            inpage = 0;
            ++col;
          }
        }
        return have;
      };

      // ---- query rows: lane r16 owns row tile * 16 + r16 = (token, head of the group)
      const int qr = tile * 16 + r16;
      const int token = qr / grp, head = kvh * grp + (qr - token * grp);
      const bool row_ok = token < n;
      const long long qrow = (long long)rank * a.rows + first + token;
      // keys below lim are seen; the arithmetic cannot overflow: len >= 0, token < n <= 2^31
      const int lim = row_ok ? (int)min((long long)len - n + token + 1, (long long)keys) : 0;
      uint4 qw[4];
      unsigned have[FNS];
      float m, l;
      f32x4_t acc[8];
      auto start = [&] {
        col = k0 * KB / a.page_size;
        inpage = k0 * KB - col * a.page_size;
        if (col < page0) take_pages(col);
#pragma unroll
        for (int i = 0; i < FNS; ++i) have[i] = copy(k0 + i, i);
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) acc[dt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
      };
      start();
      const bf16_t* src = q + (row_ok ? qrow * a.ld_q + head * PHD : 0);   // rows of nobody: any row, they see no key
#pragma unroll
      for (int t = 0; t < 4; ++t)
        qw[t] = *reinterpret_cast<const uint4*>(src + (E4M3 ? 16 * g + 8 * (t & 1) + 64 * (t >> 1) : 32 * t + 8 * g));
      bf16x8_t qf[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        asm volatile("" : "+v"(qw[t].x), "+v"(qw[t].y), "+v"(qw[t].z), "+v"(qw[t].w));   // the wait for q stands in front of the loop
        qf[t] = __builtin_bit_cast(bf16x8_t, qw[t]);
      }
      const float sc_log2 = E4M3 && a.k_scale ? scale_log2 * a.k_scale[h] : scale_log2;

      auto sweep = [&](auto fp32_c) {            // the first FNS copies are under way
        int slot = 0;
        for (int blk = k0; blk < k1; ++blk) {
          wait_vmcnt<(FNS - 1) * FNI>();         // this block has landed; the next one may be in flight
          const uint4* ks = mine + slot * (FNI * 64);
          const uint4* vs = ks + 4 * 64;
          const unsigned pg = have[0];
          // K: lane r16 = key of the group, dims as q's; V: keys 4 g .. 4 g + 3 of the group, one dim (two in e4m3)
          uint4 kw[4];
          uint2 vw[8];
          const int vr = 4 * g + (r16 >> 2);
          if constexpr (E4M3) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int c = 0; c < 2; ++c) kw[j * 2 + c] = ks[(j * 16 + r16) * CPR + ((c * 4 + g) ^ fk_swz<true>(r16))];
            const lds_c_t va = (lds_c_t)vs + vr * 128 + (r16 & 1) * 8;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
              for (int dt = 0; dt < 4; ++dt)
                vw[j * 4 + dt] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (lds_s4_t)(va + j * 16 * 128 + (((dt * 2 + ((r16 & 3) >> 1)) ^ fv_swz<true>(vr)) << 4))));
          } else {
#pragma unroll
            for (int t = 0; t < 4; ++t) kw[t] = ks[r16 * CPR + ((t * 4 + g) ^ fk_swz<false>(r16))];
            const lds_c_t va = (lds_c_t)vs + vr * 256 + (r16 & 1) * 8;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt)
              vw[dt] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                  (lds_s4_t)(va + (((dt * 2 + ((r16 & 3) >> 1)) ^ fv_swz<false>(vr)) << 4))));
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) asm volatile("" : "+v"(kw[t].x), "+v"(kw[t].y), "+v"(kw[t].z), "+v"(kw[t].w));
#pragma unroll
          for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(vw[i].x), "+v"(vw[i].y));
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the fragments are in registers before the slot is filled again
          have[0] = have[1];
          have[1] = copy(blk + FNS, slot);
          slot ^= 1;
          f32x4_t sc[HV];
#pragma unroll
          for (int j = 0; j < HV; ++j) {
            sc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              uint4 kf;
              if constexpr (E4M3) {
                const uint4 w = kw[j * 2 + (t >> 1)];
                const unsigned w0 = t & 1 ? w.z : w.x, w1 = t & 1 ? w.w : w.y;
                kf = make_uint4(fp8_lo(w0), fp8_hi(w0), fp8_lo(w1), fp8_hi(w1));
              } else {
                kf = kw[t];
              }
              sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf), qf[t], sc[j], 0, 0, 0);
            }
          }
          // scores of query row r16 and keys blk * KB + 16 j + 4 g + i
          float p[HV][4], mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < HV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = blk * KB + 16 * j + 4 * g + i;
              p[j][i] = key < lim && (pg >> j & 1) ? sc[j][i] * sc_log2 : -INFINITY;
              mx = fmaxf(mx, p[j][i]);
            }
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
          const float m_new = fmaxf(m, mx);
          const float mb = m_new == -INFINITY ? 0.0f : m_new;   // no key seen so far: nothing is added
          const float alpha = __builtin_amdgcn_exp2f(m - mb);
          float sum = 0.0f;
#pragma unroll
          for (int j = 0; j < HV; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              p[j][i] = __builtin_amdgcn_exp2f(p[j][i] - mb);
              sum += p[j][i];
            }
          l = l * alpha + sum;
          m = m_new;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[dt][r] *= alpha;
          if constexpr (decltype(fp32_c)::value) {
#pragma unroll
            for (int i = 0; i < 4; ++i)          // step i of the product: the keys 4 g + i, g = 0 .. 3 (bf16 caches only)
#pragma unroll
              for (int dt = 0; dt < 8; ++dt) {
                const unsigned w = i & 2 ? vw[dt].y : vw[dt].x;
                acc[dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(i & 1 ? hi_bf(w) : lo_bf(w), p[0][i], acc[dt], 0, 0, 0);
              }
          } else {
            unsigned hi[HV][2], lo[HV][2];
#pragma unroll
            for (int j = 0; j < HV; ++j)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                hi[j][i] = pack2bf(p[j][2 * i], p[j][2 * i + 1]);
                lo[j][i] = pack2bf(p[j][2 * i] - lo_bf(hi[j][i]), p[j][2 * i + 1] - hi_bf(hi[j][i]));
              }
            if constexpr (E4M3) {                // the 32 keys' first parts, then their second
              const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0][0], hi[0][1], hi[1][0], hi[1][1]));
              const bf16x8_t pl = __builtin_bit_cast(bf16x8_t, make_uint4(lo[0][0], lo[0][1], lo[1][0], lo[1][1]));
#pragma unroll
              for (int dt = 0; dt < 4; ++dt) {   // dims 32 dt + 2 r16 (acc[2 dt]) and + 1
                unsigned ev[4], od[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                  const unsigned w = c == 0 ? vw[dt].x : c == 1 ? vw[dt].y : c == 2 ? vw[4 + dt].x : vw[4 + dt].y;
                  const unsigned s = __builtin_amdgcn_perm(w, w, 0x03010200u);   // bytes: even dim of two keys, odd dim
                  ev[c] = fp8_lo(s);
                  od[c] = fp8_hi(s);
                }
                const bf16x8_t ve = __builtin_bit_cast(bf16x8_t, make_uint4(ev[0], ev[1], ev[2], ev[3]));
                const bf16x8_t vd = __builtin_bit_cast(bf16x8_t, make_uint4(od[0], od[1], od[2], od[3]));
                acc[2 * dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, ph, acc[2 * dt], 0, 0, 0);
                acc[2 * dt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vd, ph, acc[2 * dt + 1], 0, 0, 0);
                acc[2 * dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, pl, acc[2 * dt], 0, 0, 0);
                acc[2 * dt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vd, pl, acc[2 * dt + 1], 0, 0, 0);
              }
            } else {                             // one product takes both parts against the values twice
              const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0][0], hi[0][1], lo[0][0], lo[0][1]));
#pragma unroll
              for (int dt = 0; dt < 8; ++dt) {
                const bf16x8_t v2 = __builtin_bit_cast(bf16x8_t, make_uint4(vw[dt].x, vw[dt].y, vw[dt].x, vw[dt].y));
                acc[dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v2, pf, acc[dt], 0, 0, 0);
              }
            }
          }
        }
      };
      sweep(std::false_type{});
      wait_vmcnt<0>();                           // the copies past the end write zeros: let them land
      if constexpr (!E4M3) {
        bool odd = false;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt)
#pragma unroll
          for (int r = 0; r < 4; ++r) odd |= !(fabsf(acc[dt][r]) < INFINITY);
        if (__any(odd)) {
          start();
          sweep(std::true_type{});
          wait_vmcnt<0>();
        }
      }
      l += __shfl_xor(l, 16, 64);
      l += __shfl_xor(l, 32, 64);

      // ---- dims that a lane holds: 16 dt + 4 g + r of acc[dt][r]; e4m3: 32 (dt / 2) + 8 g + 2 r + dt % 2
      auto at_dim = [&](int dt, int r) { return E4M3 ? 32 * (dt >> 1) + 8 * g + 2 * r + (dt & 1) : 16 * dt + 4 * g + r; };
      const long long unit = base + u * nb;      // place of the unit's first block
      const long long wg0 = (long long)blockIdx.x * FNW * per;
      if (from == 0 && to == nb) {
        if (row_ok) {
          const float inv = l == 0.0f ? 0.0f : (E4M3 && a.v_scale ? a.v_scale[h] : 1.0f) / l;
          bf16_t* dst = out + (qrow * a.hpr + head) * PHD;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            if constexpr (E4M3) {
              uint4 w;
              w.x = pack2bf(acc[2 * t][0] * inv, acc[2 * t + 1][0] * inv);
              w.y = pack2bf(acc[2 * t][1] * inv, acc[2 * t + 1][1] * inv);
              w.z = pack2bf(acc[2 * t][2] * inv, acc[2 * t + 1][2] * inv);
              w.w = pack2bf(acc[2 * t][3] * inv, acc[2 * t + 1][3] * inv);
              *reinterpret_cast<uint4*>(dst + 32 * t + 8 * g) = w;
            } else {
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const int dt = 2 * t + k;
                uint2 w;
                w.x = pack2bf(acc[dt][0] * inv, acc[dt][1] * inv);
                w.y = pack2bf(acc[dt][2] * inv, acc[dt][3] * inv);
                *reinterpret_cast<uint2*>(dst + 16 * dt + 4 * g) = w;
              }
            }
          }
        }
      } else {
        if (from == 0) join = FewJoin{min(16, n * grp - tile * 16), rank, kvh, first, tile, 0, unit, unit + nb, per};
        // all four stretches lie inside the unit: joined here, one partial result for the workgroup
        const bool together = unit <= wg0 && wg0 + FNW * per <= unit + nb;
        float* po = together ? reinterpret_cast<float*>(ring) + wave * FSLOT : part + (2LL * wid + (x == x0 ? 0 : 1)) * FSLOT;
        if (together) __syncthreads();           // before the partial results take the rings' place
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) {
          if constexpr (E4M3) {
            if (dt & 1) continue;
            *reinterpret_cast<f32x4_t*>(po + r16 * FPR + at_dim(dt, 0)) = f32x4_t{acc[dt][0], acc[dt + 1][0], acc[dt][1], acc[dt + 1][1]};
            *reinterpret_cast<f32x4_t*>(po + r16 * FPR + at_dim(dt, 2)) = f32x4_t{acc[dt][2], acc[dt + 1][2], acc[dt][3], acc[dt + 1][3]};
          } else {
            *reinterpret_cast<f32x4_t*>(po + r16 * FPR + at_dim(dt, 0)) = acc[dt];
          }
        }
        if (!together) {
          if (g == 0) {
            po[r16 * FPR + PHD] = m;
            po[r16 * FPR + PHD + 1] = l;
          }
        } else {
          if (g == 0) {
            s_m[wave][r16] = m;
            s_l[wave][r16] = l;
          }
          __syncthreads();
          const float* pr = reinterpret_cast<const float*>(ring);
          float* dst = part + 2LL * blockIdx.x * FNW * FSLOT;
          const int rows = min(16, n * grp - tile * 16);
          for (int i = threadIdx.x; i < rows * PHD; i += 64 * FNW) {
            const int r = i / PHD, d = i - r * PHD;
            float M = s_m[0][r];
#pragma unroll
            for (int w = 1; w < FNW; ++w) M = fmaxf(M, s_m[w][r]);
            const float mb = M == -INFINITY ? 0.0f : M;
            float num = 0.0f, den = 0.0f;
#pragma unroll
            for (int w = 0; w < FNW; ++w) {
              const float f = __builtin_amdgcn_exp2f(s_m[w][r] - mb);
              num += pr[w * FSLOT + r * FPR + d] * f;
              den += s_l[w][r] * f;
            }
            dst[r * FPR + d] = num;
            if (d == 0) {
              dst[r * FPR + PHD] = M;
              dst[r * FPR + PHD + 1] = den;
            }
          }
        }
      }
      // ---- the next unit
      x += to - from;
      if (x < x1 && x >= base + work * heads) {
        base += work * heads;
        do {                                     // (some sequence behind this one has work: x < total)
          ++b;
          if (b >= sq.at + 64) sq = load_seqs(b);
        } while (__builtin_amdgcn_readlane(sq.n, b - sq.at) == 0);
      }
    }
  }
  if (joins && lane == 0) joins[wid] = join;
}

// Joins the partial results of the units that cross stretches: a wave per (unit, row); blockIdx.x is the wave in which the unit
// begins.  Their order is that of the keys: single waves up to the first whole workgroup, the workgroups, single waves.
__global__ __launch_bounds__(64) void paged_few_join_kernel(const PagedArgs a, const float* __restrict__ part, const FewJoin* __restrict__ joins,
                                                            bf16_t* __restrict__ out) {
  const FewJoin j = joins[blockIdx.x];
  if ((int)blockIdx.y >= j.rows) return;
  const int lane = threadIdx.x;
  const long long per = j.per;
  const int w0 = blockIdx.x, w1 = (int)((j.end - 1) / per);                       // waves of the unit
  const int ga = (int)((j.begin + FNW * per - 1) / (FNW * per)), gb = (int)(j.end / (FNW * per));   // workgroups inside it
  const int head = gb > ga ? ga * FNW - w0 : w1 + 1 - w0, mid = gb > ga ? gb - ga : 0;
  const int tail = gb > ga ? w1 + 1 - gb * FNW : 0, count = head + mid + tail;
  auto slot = [&](int i) -> long long {
    if (i < head) return 2LL * (w0 + i) + ((w0 + i) * per < j.begin ? 1 : 0);
    if (i < head + mid) return 2LL * FNW * (ga + i - head);
    return 2LL * (gb * FNW + i - head - mid);
  };
  const int grp = a.hpr / a.kvpr;
  for (int r = blockIdx.y; r < j.rows; r += gridDim.y) {
    float M = -INFINITY, den = 0.0f, n0 = 0.0f, n1 = 0.0f;
    for (int c0 = 0; c0 < count; c0 += 64) {
      float pm = -INFINITY, pl = 0.0f;
      long long at = 0;
      if (c0 + lane < count) {
        at = slot(c0 + lane) * FSLOT + r * FPR;
        pm = part[at + PHD];
        pl = part[at + PHD + 1];
      }
      float mx = pm;
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
      const float m_new = fmaxf(M, mx), mb = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(M - mb), f = __builtin_amdgcn_exp2f(pm - mb);
      float sum = pl * f;
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
      den = den * alpha + sum;
      n0 *= alpha;
      n1 *= alpha;
      M = m_new;
      const int here = min(64, count - c0);
      for (int i0 = 0; i0 < here; i0 += 8) {
        float2 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
          v[i] = i0 + i < here ? *reinterpret_cast<const float2*>(part + lane64(at, i0 + i) + lane * 2) : make_float2(0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i0 + i));   // 0 behind the last
          n0 += v[i].x * fi;
          n1 += v[i].y * fi;
        }
      }
    }
    const int qr = j.tile * 16 + r, token = qr / grp, h = j.kvh * grp + (qr - token * grp);
    const float inv = den == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[j.rank * a.kvpr + j.kvh] : 1.0f) / den;
    *reinterpret_cast<unsigned*>(out + (((long long)j.rank * a.rows + j.first + token) * a.hpr + h) * PHD + lane * 2) = pack2bf(n0 * inv, n1 * inv);
  }
}

size_t paged_few_workspace_bytes() {
  return (size_t)FMAX_WGS * FNW * (sizeof(FewJoin) + 2 * FSLOT * sizeof(float));
}

hipError_t launch_paged_few(const PagedArgs& a, int e4m3, int max_new, const bf16_t* q, bf16_t* out, const void* kc, const void* vc,
                            void* workspace, hipStream_t s) {
  const long long grp = a.hpr / a.kvpr, cap = (long long)a.max_pages * a.page_size;
  const long long kb = e4m3 ? 32 : 16, nb = (cap + kb - 1) / kb;
  const int whole = nb <= 4;                     // caches of so few keys are not worth a second kernel
  const int least = whole ? 1 : 2;
  const long long most = ((a.rows * grp + 15) / 16 + a.batch) * a.T * a.kvpr * (whole ? 1 : nb);   // blocks, at most
  const int wgs = (int)std::min<long long>(FMAX_WGS, (most + least * FNW - 1) / (least * FNW));
  FewJoin* joins = reinterpret_cast<FewJoin*>(workspace);
  float* part = reinterpret_cast<float*>(joins + FMAX_WGS * FNW);
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)PHD);
  auto kernel = e4m3 ? paged_few_kernel<true> : paged_few_kernel<false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(64 * FNW), 0, s, a, q, out, kc, vc, part, whole ? nullptr : joins, scale_log2,
                     least, whole);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || whole) return e;
  const int rows = (int)std::min<long long>(16, grp * max_new);
  hipLaunchKernelGGL(paged_few_join_kernel, dim3((unsigned)(wgs * FNW), (unsigned)rows), dim3(64), 0, s, a, part, joins, out);
  return hipGetLastError();
}

}  // namespace caat
