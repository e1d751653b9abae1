// Attention of few new tokens per sequence (decode steps, drafted tokens) over a paged key / value cache, gfx950.
//
// What bounds it: the K / V rows, read once from HBM.  The unit of work is one or two tiles of 16 (token, query head of the group)
// rows of one sequence, rank and key / value head, times a block of keys (16 in bf16, 32 in e4m3: 8 KB of K and V).  The blocks of
// all units stand in one line, sequence by sequence, and every WAVE of the launch takes an equal stretch of it, so a batch of
// one long and many short sequences fills the chip like an even one, whatever the lengths (which only the device
// knows).  A wave copies its blocks global -> LDS into two slots that only it reads, waits for its own copies alone, and computes
// S = K q^T and O^T += V^T P with MFMAs (columns = query rows; most are idle for multi-head attention, but the matrix unit has
// nothing else to do).  P goes in as an exact sum of three bf16 values, as in the contiguous decode (two of them, 16 bits, us: 300 keys
// of one sequence 10.1 and not 10.4, 64 x 2048 323 and 323, e4m3 63 of up to 8191 49.8 and 50.2); a wave whose sums are not finite
// (infinity times a part that is zero, or times the zero of a row that does not see the key) repeats its keys with fp32 MFMAs, and
// those that some of its rows do not see without.  A unit inside one stretch is finished there; of
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

// What the wave in which a unit begins says about it.  They stand in the order of the units where the launch cannot have more
// units than waves, in that of the waves (of which one begins at most one unit that it does not finish) otherwise.
struct FewJoin {
  int rows;                                      // 0: the unit was finished by that wave
  int rank, kvh, first, row0;                    // row0: the unit's first (token, head) row of the sequence
  int begin, end, per;                           // the unit's blocks in the line of all of them; length of a stretch, negative:
                                                 // of a workgroup
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
  int units, work;                               // of one (rank, key / value head): units and their length in the line
};

// How the units are dealt out.  FEW_LINE: as the head of this file says.  FEW_WAVE: whole units to waves, FEW_WG: a unit to a
// workgroup; neither leaves anything for the second kernel.
enum FewMode { FEW_LINE = 0, FEW_WAVE = 1, FEW_WG = 2 };
// A unit's start (its queries' and pages' way, the first block's, its results) takes a wave about as long as FSTART blocks: they
// stand in the line in front of the unit's own.  Where units have FWIDE blocks and more on average, a stretch belongs to a workgroup,
// whose waves take a quarter of a unit's blocks each and join their results in LDS, so that a quarter as many go through the
// workspace (us, a wave's stretches / a workgroup's: 32 heads, 63 x 2048 keys 370 / 327, 128 x 512 171 / 173, 128 x 256 89 / 100;
// 64 / 8 heads, 48 of up to 16384 145 / 144; 58 of 19 under a table of 640, 16 heads 13.7 / 15.6).
static constexpr int FSTART = 3;
static constexpr int FWIDE = 24;

// NT: tiles of 16 query rows of a unit, which share the fragments of K and V
template <bool E4M3, int NT>
__global__ __launch_bounds__(64 * FNW, 2) void paged_few_kernel(const PagedArgs a, const bf16_t* __restrict__ q, bf16_t* __restrict__ out,
                                                             const void* __restrict__ kc, const void* __restrict__ vc,
                                                             float* __restrict__ part, FewJoin* __restrict__ joins, float scale_log2,
                                                             int least, int mode, int unit_joins) {
  constexpr int KB = E4M3 ? 32 : 16;             // keys per block
  constexpr int HV = KB / 16;                    // groups of 16 keys, each inside one page
  constexpr int ELT = E4M3 ? 1 : 2;
  constexpr int RPC = 1024 / (PHD * ELT);        // rows per copy: 4 or 8
  constexpr int CPR = 64 / RPC;                  // 16-byte chunks per row
  constexpr int ROWS = 16 * NT;                  // query rows of a unit
  constexpr long long FSLOT = ROWS * FPR;        // floats of a partial result
  __shared__ uint4 ring[FNW * FNS * FNI * 64];
  static_assert(FNW * 16 * FPR * 4 <= FNW * FNS * FNI * 1024, "the partial results take the rings' place");
  __shared__ float s_m[FNW][16], s_l[FNW][16];
  const int lane = threadIdx.x & 63;
  const int wave = uni(threadIdx.x >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int grp = a.hpr / a.kvpr, heads = a.T * a.kvpr;
  const int wid = blockIdx.x * FNW + wave;
  const int cap = a.max_pages * a.page_size;

  // ---- the line of all blocks, and this wave's stretch of it
  auto load_seqs = [&](int at, int start_blocks) {
    SeqChunk c;
    c.at = at;
    const int b = min(at + lane, a.batch - 1);   // (no branch: several chunks' loads are under way at once)
    c.n = at + lane < a.batch ? seq_rows(a, b, c.first) : 0;
    c.len = max(a.lens[b], 0);
    const int nb = mode == FEW_LINE ? (min(c.len, cap) + KB - 1) / KB + start_blocks : 1;
    c.units = (int)(((long long)c.n * grp + ROWS - 1) / ROWS);
    c.work = c.units * nb;
    return c;
  };
  SeqChunk sq = load_seqs(0, 0);
  int units_to = wave_sums(sq.units), work_to = wave_sums(sq.work);
  int units = __builtin_amdgcn_readlane(units_to, 63), total = __builtin_amdgcn_readlane(work_to, 63);
  int chunk_units = lane ? 0 : units, chunk_work = lane ? 0 : total;   // lane k: of chunk k, the first 64 of them
  bool beyond = (work_to | units_to) < 0;                     // a sum has passed 31 bits (one sequence cannot)
  for (int at = 64; at < a.batch; at += 256) {
    SeqChunk c[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) c[k] = load_seqs(at + 64 * k, 0);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int usums = wave_sums(c[k].units), wsums = wave_sums(c[k].work);
      const int u = __builtin_amdgcn_readlane(usums, 63), w = __builtin_amdgcn_readlane(wsums, 63);
      units += u;
      total += w;
      beyond |= (usums | wsums | units | total) < 0;
      if (lane == at / 64 + k) {
        chunk_units = u;
        chunk_work = w;
      }
    }
  }
  const bool wide = mode == FEW_WG || (mode == FEW_LINE && total >= (long long)units * FWIDE);
  const int start_blocks = mode == FEW_LINE ? (wide ? FSTART * FNW : FSTART) : 0;
  // The host has checked that the line has less than 2^31 places.  A list that gives rows to many sequences can make it longer: then
  // nobody takes any.
  const long long line = ((long long)units * start_blocks + total) * heads;
  const bool none = __any(beyond) || line > 0x7FFFFFFF;
  total = none ? 0 : (int)line;
  units = none ? 0 : units * heads;
  sq.work += sq.units * start_blocks;
  work_to += units_to * start_blocks;
  const int takers = wide ? gridDim.x : gridDim.x * FNW, taker = wide ? blockIdx.x : wid;
  const int per = mode == FEW_WG ? 1 : max((int)((unsigned)(total + takers - 1) / (unsigned)takers), wide ? least * FNW : least);
  const int x0 = (int)min((long long)taker * per, (long long)total), x1 = min(total - x0, per) + x0;
  FewJoin join = {};
  if (x0 < x1) {
    // the sequence of place x0: `base` is where its first unit begins, unit0 the number of that unit
    int b = a.batch, unit0 = 0, base = 0;
    if (a.batch > 64) {                          // its chunk, or the last of the first 64
      const int own = chunk_work + chunk_units * start_blocks, upto = wave_sums(own), uupto = wave_sums(chunk_units);
      const unsigned long long over = __ballot(upto * heads > x0);
      const int k = over ? __builtin_ctzll(over) : 63;
      if (k > 0) {
        base = __builtin_amdgcn_readlane(upto - own, k) * heads;
        unit0 = __builtin_amdgcn_readlane(uupto - chunk_units, k) * heads;
        sq = load_seqs(64 * k, start_blocks);
        work_to = wave_sums(sq.work);
        units_to = wave_sums(sq.units);
      }
    }
    while (sq.at < a.batch) {
      const unsigned long long over = __ballot(base + work_to * heads > x0);
      if (over) {
        b = __builtin_ctzll(over);
        base += __builtin_amdgcn_readlane(work_to - sq.work, b) * heads;
        unit0 += __builtin_amdgcn_readlane(units_to - sq.units, b) * heads;
        b += sq.at;
        break;
      }
      base += __builtin_amdgcn_readlane(work_to, 63) * heads;
      unit0 += __builtin_amdgcn_readlane(units_to, 63) * heads;
      sq = load_seqs(sq.at + 64, start_blocks);
      work_to = wave_sums(sq.work);
      units_to = wave_sums(sq.units);
    }
    int pages = -1, page0 = -1, pages_of = -1;   // lane l: entry page0 + l of sequence pages_of's table, -1: no page
    uint4* mine = ring + wave * (FNS * FNI * 64);

    for (int x = x0; x < x1 && b < a.batch;) {
      const int sl = b - sq.at;
      const int n = __builtin_amdgcn_readlane(sq.n, sl), first = __builtin_amdgcn_readlane(sq.first, sl);
      const int len = __builtin_amdgcn_readlane(sq.len, sl), work = __builtin_amdgcn_readlane(sq.work, sl);
      const int tiles = __builtin_amdgcn_readlane(sq.units, sl);
      const int keys = min(len, cap);
      const int nblk = (keys + KB - 1) / KB;     // may be 0
      const int nb = mode == FEW_LINE ? nblk + start_blocks : 1;
      const int u = (int)((unsigned)(x - base) / (unsigned)nb);
      const int unit = base + u * nb;            // place of the unit
      const int to = min(unit + nb, x1);         // and of the stretch's part of it: x .. to - 1
      const int h = (int)((unsigned)u / (unsigned)tiles), tile = u - h * tiles;
      const int rank = h / a.kvpr, kvh = h - rank * a.kvpr;
      // its blocks of keys
      int k0 = 0, k1 = nblk;
      if (mode == FEW_LINE) {
        k0 = max(x - unit - start_blocks, 0);
        k1 = max(to - unit - start_blocks, 0);
        if (to < unit + nb && k1 == 0) break;    // the stretch ends in front of the first one
      }
      if (wide) {
        const int all = k1 - k0, from = k0;
        k0 = from + (int)((long long)all * wave / FNW);
        k1 = from + (int)((long long)all * (wave + 1) / FNW);
      }
      const bool begins = unit + start_blocks >= x0;   // its first block lies in this stretch
      const bool all_here = begins && to == unit + nb;

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

      // ---- query rows: lane r16 owns rows tile * ROWS + 16 nt + r16 = (token, head of the group)
      bool row_ok[NT];
      int lim[NT];                               // keys below are seen
      long long qat[NT];                         // (rank's row) * heads + head
      bf16x8_t qf[NT][4];
      unsigned have[FNS];
      float m[NT], l[NT];
      f32x4_t acc[NT][8];
      auto start = [&] {
        col = k0 * KB / a.page_size;
        inpage = k0 * KB - col * a.page_size;
        if (col < page0) take_pages(col);
#pragma unroll
        for (int i = 0; i < FNS; ++i) have[i] = copy(k0 + i, i);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          m[nt] = -INFINITY;
          l[nt] = 0.0f;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) acc[nt][dt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
      };
      start();
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int qr = tile * ROWS + nt * 16 + r16;
        const int token = qr / grp, head = kvh * grp + (qr - token * grp);
        const long long qrow = (long long)rank * a.rows + first + token;
        row_ok[nt] = token < n;
        lim[nt] = row_ok[nt] ? min(len - n + token + 1, keys) : 0;   // (len >= 0 and token < n: no overflow)
        qat[nt] = qrow * a.hpr + head;
        const bf16_t* src = q + (row_ok[nt] ? qrow * a.ld_q + head * PHD : 0);   // rows of nobody: any row, they see no key
        uint4 qw[4];
#pragma unroll
        for (int t = 0; t < 4; ++t)
          qw[t] = *reinterpret_cast<const uint4*>(src + (E4M3 ? 16 * g + 8 * (t & 1) + 64 * (t >> 1) : 32 * t + 8 * g));
#pragma unroll
        for (int t = 0; t < 4; ++t) qf[nt][t] = __builtin_bit_cast(bf16x8_t, qw[t]);
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int t = 0; t < 4; ++t) asm volatile("" : "+v"(qf[nt][t]));   // the wait for q stands in front of the loop
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
          uint4 kf[HV][4];                       // dims of step t, for all query tiles
#pragma unroll
          for (int j = 0; j < HV; ++j)
#pragma unroll
            for (int t = 0; t < 4; ++t) {
              if constexpr (E4M3) {
                const uint4 w = kw[j * 2 + (t >> 1)];
                const unsigned w0 = t & 1 ? w.z : w.x, w1 = t & 1 ? w.w : w.y;
                kf[j][t] = make_uint4(fp8_lo(w0), fp8_hi(w0), fp8_lo(w1), fp8_hi(w1));
              } else {
                kf[j][t] = kw[t];
              }
            }
          // scores of query row r16 of tile nt and keys blk * KB + 16 j + 4 g + i, then their probabilities in three parts
          unsigned hi[NT][HV][2], mid[NT][HV][2], lo[NT][HV][2];
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            f32x4_t sc[HV];
#pragma unroll
            for (int j = 0; j < HV; ++j) {
              sc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
              for (int t = 0; t < 4; ++t)
                sc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, kf[j][t]), qf[nt][t], sc[j], 0, 0, 0);
            }
            float p[HV][4], mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < HV; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int key = blk * KB + 16 * j + 4 * g + i;
                p[j][i] = key < lim[nt] && (pg >> j & 1) ? sc[j][i] * sc_log2 : -INFINITY;
                mx = fmaxf(mx, p[j][i]);
              }
            mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = fmaxf(m[nt], mx);
            const float mb = m_new == -INFINITY ? 0.0f : m_new;   // no key seen so far: nothing is added
            if (__any(m_new != m[nt])) {         // the running maximum settles after the first blocks
              const float alpha = __builtin_amdgcn_exp2f(m[nt] - mb);
              l[nt] *= alpha;
#pragma unroll
              for (int dt = 0; dt < 8; ++dt)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[nt][dt][r] *= alpha;
              m[nt] = m_new;
            }
#pragma unroll
            for (int j = 0; j < HV; ++j)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                p[j][i] = __builtin_amdgcn_exp2f(p[j][i] - mb);
                l[nt] += p[j][i];
              }
#pragma unroll
            for (int j = 0; j < HV; ++j)
#pragma unroll
              for (int i = 0; i < 2; ++i) {
                const float p0 = p[j][2 * i], p1 = p[j][2 * i + 1];
                hi[nt][j][i] = pack2bf(p0, p1);
                const float r0 = p0 - lo_bf(hi[nt][j][i]), r1 = p1 - hi_bf(hi[nt][j][i]);   // exact, as is the next difference
                mid[nt][j][i] = pack2bf(r0, r1);
                lo[nt][j][i] = pack2bf(r0 - lo_bf(mid[nt][j][i]), r1 - hi_bf(mid[nt][j][i]));
              }
            if constexpr (decltype(fp32_c)::value) {
#pragma unroll
              for (int i = 0; i < 4; ++i)        // step i of the product: the keys 4 g + i, g = 0 .. 3
#pragma unroll
                for (int dt = 0; dt < 8; ++dt) {
                  const unsigned w = i & 2 ? vw[dt].y : vw[dt].x;
                  acc[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x4f32(i & 1 ? hi_bf(w) : lo_bf(w), p[0][i], acc[nt][dt], 0, 0, 0);
                }
            } else if constexpr (!E4M3) {        // one product takes the first two parts against the values twice
              const bf16x8_t pf = __builtin_bit_cast(bf16x8_t, make_uint4(hi[nt][0][0], hi[nt][0][1], mid[nt][0][0], mid[nt][0][1]));
              const short4_t pl = __builtin_bit_cast(short4_t, make_uint2(lo[nt][0][0], lo[nt][0][1]));
#pragma unroll
              for (int dt = 0; dt < 8; ++dt) {
                const bf16x8_t v2 = __builtin_bit_cast(bf16x8_t, make_uint4(vw[dt].x, vw[dt].y, vw[dt].x, vw[dt].y));
                acc[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v2, pf, acc[nt][dt], 0, 0, 0);
              }
#pragma unroll
              for (int dt = 0; dt < 8; ++dt)
                acc[nt][dt] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(short4_t, vw[dt]), pl, acc[nt][dt], 0, 0, 0);
            }
          }
          if constexpr (E4M3) {                  // the 32 keys' first parts, their second, their third
#pragma unroll
            for (int dt = 0; dt < 4; ++dt) {     // dims 32 dt + 2 r16 (acc[2 dt]) and + 1
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
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                const bf16x8_t ph = __builtin_bit_cast(bf16x8_t, make_uint4(hi[nt][0][0], hi[nt][0][1], hi[nt][HV - 1][0], hi[nt][HV - 1][1]));
                const bf16x8_t pm = __builtin_bit_cast(bf16x8_t, make_uint4(mid[nt][0][0], mid[nt][0][1], mid[nt][HV - 1][0], mid[nt][HV - 1][1]));
                const bf16x8_t pl = __builtin_bit_cast(bf16x8_t, make_uint4(lo[nt][0][0], lo[nt][0][1], lo[nt][HV - 1][0], lo[nt][HV - 1][1]));
                acc[nt][2 * dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, ph, acc[nt][2 * dt], 0, 0, 0);
                acc[nt][2 * dt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vd, ph, acc[nt][2 * dt + 1], 0, 0, 0);
                acc[nt][2 * dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, pm, acc[nt][2 * dt], 0, 0, 0);
                acc[nt][2 * dt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vd, pm, acc[nt][2 * dt + 1], 0, 0, 0);
                acc[nt][2 * dt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ve, pl, acc[nt][2 * dt], 0, 0, 0);
                acc[nt][2 * dt + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vd, pl, acc[nt][2 * dt + 1], 0, 0, 0);
              }
            }
          }
        }
      };
      sweep(std::false_type{});
      wait_vmcnt<0>();                           // the copies past the end write zeros: let them land
      // A value that is not finite, times a probability of zero: of a later part, or of a row that does not see its key (one new
      // token has no such rows).  Then the blocks that every row sees are done again with whole probabilities, and the other keys by
      // lanes, each for its row and dims.
      const int cut = max(k0, min(k1, max(min(len - n + tile * ROWS / grp + 1, keys), 0) / KB));
      if (!E4M3 || cut < k1) {
        bool odd = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int dt = 0; dt < 8; ++dt)
#pragma unroll
            for (int r = 0; r < 4; ++r) odd |= !(fabsf(acc[nt][dt][r]) < INFINITY);
        if (__any(odd)) {
          const int to_key = min(k1 * KB, keys);
          k1 = cut;
          start();
          sweep(std::integral_constant<bool, !E4M3>{});
          wait_vmcnt<0>();
          for (int key = cut * KB; key < to_key; ++key) {
            const int kcol = key / a.page_size, page = a.table[(long long)b * a.max_pages + kcol];
            if (page < 0 || page >= a.n_pages) continue;
            const long long at = (page * a.s_page + (key - kcol * a.page_size) * a.s_row) * ELT;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              float s = 0.0f;
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                uint4 kw;
                if constexpr (E4M3) {
                  const uint2 w = *reinterpret_cast<const uint2*>(kh + at + 16 * g + 8 * (t & 1) + 64 * (t >> 1));
                  kw = make_uint4(fp8_lo(w.x), fp8_hi(w.x), fp8_lo(w.y), fp8_hi(w.y));
                } else {
                  kw = *reinterpret_cast<const uint4*>(kh + at + (32 * t + 8 * g) * 2);
                }
                s += dot8(kw, __builtin_bit_cast(uint4, qf[nt][t]));
              }
              s += __shfl_xor(s, 16, 64);
              s += __shfl_xor(s, 32, 64);
              if (key >= lim[nt]) continue;
              s *= sc_log2;
              asm volatile("" : "+v"(s));        // its rounding, which m_new has too, stays in front of the difference
              const float m_new = fmaxf(m[nt], s), mb = m_new == -INFINITY ? 0.0f : m_new;
              const float alpha = __builtin_amdgcn_exp2f(m[nt] - mb), p = __builtin_amdgcn_exp2f(s - mb);
              m[nt] = m_new;
              l[nt] = l[nt] * alpha + (g == 0 ? p : 0.0f);
#pragma unroll
              for (int t = 0; t < 4; ++t) {
                uint4 w;                         // dims of acc[2 t] and acc[2 t + 1]: e4m3 in turn, bf16 one after the other
                if constexpr (E4M3) {
                  const uint2 c = *reinterpret_cast<const uint2*>(vh + at + 32 * t + 8 * g);
                  w = make_uint4(fp8_lo(c.x), fp8_hi(c.x), fp8_lo(c.y), fp8_hi(c.y));
                } else {
                  const uint2 c = *reinterpret_cast<const uint2*>(vh + at + (32 * t + 4 * g) * 2);
                  const uint2 d = *reinterpret_cast<const uint2*>(vh + at + (32 * t + 16 + 4 * g) * 2);
                  w = make_uint4(c.x, c.y, d.x, d.y);
                }
                const float v[8] = {lo_bf(w.x), hi_bf(w.x), lo_bf(w.y), hi_bf(w.y), lo_bf(w.z), hi_bf(w.z), lo_bf(w.w), hi_bf(w.w)};
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  acc[nt][2 * t][r] = acc[nt][2 * t][r] * alpha + p * v[E4M3 ? 2 * r : r];
                  acc[nt][2 * t + 1][r] = acc[nt][2 * t + 1][r] * alpha + p * v[E4M3 ? 2 * r + 1 : 4 + r];
                }
              }
            }
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        l[nt] += __shfl_xor(l[nt], 16, 64);
        l[nt] += __shfl_xor(l[nt], 32, 64);
      }

      // ---- dims that a lane holds: 16 dt + 4 g + r of acc[dt][r]; e4m3: 32 (dt / 2) + 8 g + 2 r + dt % 2
      const int rows = min(ROWS, n * grp - tile * ROWS);
      auto put = [&](float* po, const f32x4_t* c) {   // a tile's sums as fp32 rows
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const f32x4_t x = c[2 * t], y = c[2 * t + 1];
          float* at = po + r16 * FPR + 32 * t;
          if constexpr (E4M3) {
            *reinterpret_cast<f32x4_t*>(at + 8 * g) = f32x4_t{x[0], y[0], x[1], y[1]};
            *reinterpret_cast<f32x4_t*>(at + 8 * g + 4) = f32x4_t{x[2], y[2], x[3], y[3]};
          } else {
            *reinterpret_cast<f32x4_t*>(at + 4 * g) = x;
            *reinterpret_cast<f32x4_t*>(at + 16 + 4 * g) = y;
          }
        }
      };
      const float vs = E4M3 && a.v_scale ? a.v_scale[h] : 1.0f;
      if (lane == 0 && (unsigned)(unit0 + u) < (unsigned)unit_joins && begins) {
        FewJoin* j = joins + unit0 + u;
        if (all_here) j->rows = 0;
        else *j = FewJoin{rows, rank, kvh, first, tile * ROWS, unit + start_blocks, unit + nb, wide ? -per : per};
      }
      if (!wide && all_here) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (!row_ok[nt]) continue;
          float inv = vs / l[nt];
          if (l[nt] == 0.0f) {                   // no key seen, or all scores minus infinity: zeros, whatever the values hold
            inv = 0.0f;
#pragma unroll
            for (int dt = 0; dt < 8; ++dt) acc[nt][dt] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
          }
          bf16_t* dst = out + qat[nt] * PHD;
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const f32x4_t x = acc[nt][2 * t], y = acc[nt][2 * t + 1];
            if constexpr (E4M3) {
              *reinterpret_cast<uint4*>(dst + 32 * t + 8 * g) =
                  make_uint4(pack2bf(x[0] * inv, y[0] * inv), pack2bf(x[1] * inv, y[1] * inv), pack2bf(x[2] * inv, y[2] * inv),
                             pack2bf(x[3] * inv, y[3] * inv));
            } else {
              *reinterpret_cast<uint2*>(dst + 32 * t + 4 * g) = make_uint2(pack2bf(x[0] * inv, x[1] * inv), pack2bf(x[2] * inv, x[3] * inv));
              *reinterpret_cast<uint2*>(dst + 32 * t + 16 + 4 * g) = make_uint2(pack2bf(y[0] * inv, y[1] * inv), pack2bf(y[2] * inv, y[3] * inv));
            }
          }
        }
      } else {
        if (begins && !all_here && (!wide || wave == 0))
          join = FewJoin{rows, rank, kvh, first, tile * ROWS, unit + start_blocks, unit + nb, wide ? -per : per};
        const int wg0 = blockIdx.x * FNW * per;
        if (wide || (unit + start_blocks <= wg0 && wg0 + FNW * per <= unit + nb)) {
          // the workgroup's waves all work at this unit: joined here, one (partial) result
          float* po = reinterpret_cast<float*>(ring);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (nt * 16 >= rows) break;
            __syncthreads();                     // before the partial results take the rings' place, or the last tile's
            put(po + wave * 16 * FPR, acc[nt]);
            if (g == 0) {
              s_m[wave][r16] = m[nt];
              s_l[wave][r16] = l[nt];
            }
            __syncthreads();
            float* dst = part + (2LL * blockIdx.x * FNW + (wide && begins ? 1 : 0)) * FSLOT + nt * 16 * FPR;
            const int here = min(16, rows - nt * 16);
            for (int i = threadIdx.x; i < here * PHD; i += 64 * FNW) {
              const int r = i / PHD, d = i - r * PHD;
              float M = s_m[0][r];
#pragma unroll
              for (int w = 1; w < FNW; ++w) M = fmaxf(M, s_m[w][r]);
              const float mb = M == -INFINITY ? 0.0f : M;
              float num = 0.0f, den = 0.0f;
#pragma unroll
              for (int w = 0; w < FNW; ++w) {
                const float f = __builtin_amdgcn_exp2f(s_m[w][r] - mb);
                num += po[(w * 16 + r) * FPR + d] * f;
                den += s_l[w][r] * f;
              }
              if (wide && all_here) {
                const int qr = tile * ROWS + nt * 16 + r, token = qr / grp, head = kvh * grp + (qr - token * grp);
                out[(((long long)rank * a.rows + first + token) * a.hpr + head) * PHD + d] = f2bf(den == 0.0f ? 0.0f : num * (vs / den));
                continue;
              }
              dst[r * FPR + d] = num;
              if (d == 0) {
                dst[r * FPR + PHD] = M;
                dst[r * FPR + PHD + 1] = den;
              }
            }
          }
          __syncthreads();                       // before the next unit's blocks take the partial results' place
        } else {
          float* po = part + (2LL * wid + (begins ? 1 : 0)) * FSLOT;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            put(po + nt * 16 * FPR, acc[nt]);
            if (g == 0) {
              po[(nt * 16 + r16) * FPR + PHD] = m[nt];
              po[(nt * 16 + r16) * FPR + PHD + 1] = l[nt];
            }
          }
        }
      }
      // ---- the next unit
      x = to;
      if (x < x1 && x >= base + work * heads) {
        base += work * heads;
        unit0 += tiles * heads;
        while (++b < a.batch) {
          if (b >= sq.at + 64) sq = load_seqs(b, start_blocks);
          if (__builtin_amdgcn_readlane(sq.units, b - sq.at) > 0) break;
        }
      }
    }
  }
  if (unit_joins) {                              // the launch has room for unit_joins units
    for (int i = units + wid * 64 + lane; i < unit_joins; i += gridDim.x * FNW * 64) joins[i].rows = 0;
  } else if (mode == FEW_LINE && lane == 0) {
    joins[wid] = join;
  }
}

// Joins the partial results of the units that cross stretches: a wave per (unit, row).  Their order is that of the keys: single
// waves up to the first whole workgroup, the workgroups, single waves.
__global__ __launch_bounds__(64) void paged_few_join_kernel(const PagedArgs a, const float* __restrict__ part, const FewJoin* __restrict__ joins,
                                                            bf16_t* __restrict__ out, int slot_rows) {
  const FewJoin j = joins[blockIdx.x];
  if ((int)blockIdx.y >= j.rows) return;
  const int lane = threadIdx.x;
  int head, mid, tail, w0, ga = 0, gb = 0;
  if (j.per < 0) {                               // workgroups only
    w0 = j.begin / -j.per;
    head = (j.end - 1) / -j.per + 1 - w0;
    mid = tail = 0;
  } else {
    const long long wg = (long long)FNW * j.per;
    const int w1 = (j.end - 1) / j.per;
    w0 = j.begin / j.per;                        // to w1: waves of the unit
    ga = (int)((j.begin + wg - 1) / wg);         // to gb - 1: workgroups inside it
    gb = (int)(j.end / wg);
    head = gb > ga ? ga * FNW - w0 : w1 + 1 - w0;
    mid = gb > ga ? gb - ga : 0;
    tail = gb > ga ? w1 + 1 - gb * FNW : 0;
  }
  const int count = head + mid + tail;
  auto slot = [&](int i) -> long long {          // the first one's lies behind that of the unit before
    if (i < head) return 2LL * (w0 + i) * (j.per < 0 ? FNW : 1) + (i == 0 ? 1 : 0);
    if (i < head + mid) return 2LL * FNW * (ga + i - head);
    return 2LL * (gb * FNW + i - head - mid);
  };
  const int grp = a.hpr / a.kvpr;
  for (int r = blockIdx.y; r < j.rows; r += gridDim.y) {
    float M = -INFINITY, den = 0.0f, n0 = 0.0f, n1 = 0.0f;
    auto take = [&](int c0, auto most_c) {       // partial results c0 .. c0 + MOST - 1, all loads under way at once
      constexpr int MOST = decltype(most_c)::value;
      const int here = min(MOST, count - c0);
      const long long at = (slot(c0 + min(lane, here - 1)) * slot_rows + r) * FPR;
      const float2 ml = *reinterpret_cast<const float2*>(part + at + PHD);
      float2 v[MOST];
#pragma unroll
      for (int i = 0; i < MOST; ++i) v[i] = *reinterpret_cast<const float2*>(part + lane64(at, i) + lane * 2);
      const float pm = lane < here ? ml.x : -INFINITY, pl = lane < here ? ml.y : 0.0f;
      float mx = pm;
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) mx = fmaxf(mx, __shfl_xor(mx, off, 64));
      const float m_new = fmaxf(M, mx), mb = m_new == -INFINITY ? 0.0f : m_new;
      const float alpha = __builtin_amdgcn_exp2f(M - mb), f = lane < here ? __builtin_amdgcn_exp2f(pm - mb) : 0.0f;
      float sum = pl * f;
#pragma unroll
      for (int off = 32; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
      den = den * alpha + sum;
      n0 *= alpha;
      n1 *= alpha;
      M = m_new;
#pragma unroll
      for (int i = 0; i < MOST; ++i) {
        const float fi = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i));
        if (i < here) {
          n0 += v[i].x * fi;
          n1 += v[i].y * fi;
        }
      }
    };
    if (count <= 8) take(0, std::integral_constant<int, 8>{});
    else
      for (int c0 = 0; c0 < count; c0 += 32) take(c0, std::integral_constant<int, 32>{});
    const int qr = j.row0 + r, token = qr / grp, h = j.kvh * grp + (qr - token * grp);
    const float inv = den == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[j.rank * a.kvpr + j.kvh] : 1.0f) / den;
    if (den == 0.0f) n0 = n1 = 0.0f;
    *reinterpret_cast<unsigned*>(out + (((long long)j.rank * a.rows + j.first + token) * a.hpr + h) * PHD + lane * 2) = pack2bf(n0 * inv, n1 * inv);
  }
}

// Tiles of 16 query rows per unit: one read of K and V for all of them
static int few_tiles(const PagedArgs& a, int max_new) { return (long long)max_new * (a.hpr / a.kvpr) <= 16 ? 1 : 2; }

// at most as many units as this: a sequence's last tile is not full
static long long few_units(const PagedArgs& a, int nt) {
  const long long rows = (long long)a.rows * (a.hpr / a.kvpr);
  return std::min((rows + 16 * nt - 1) / (16 * nt) + a.batch - 1, rows) * a.T * a.kvpr;
}

// More than 32 rows of queries go to the prompts' kernel, whose vector work per score is less (us, here with three and four
// tiles / there: 64 / 8 heads, 24 sequences of 6000 keys, 40 rows 150 / 123, 64 rows 219 / 128; one of 40000 63 / 45, 71 / 48; 64 of
// 500 keys in e4m3, 40 rows, 60 / 22).  Two tiles stay here, whose probabilities are whole and not of 8 bits: 32 rows, here / there, 24 of
// 6000 119 / 121, e4m3 78 / 83, one of 40000 47 / 44, but 64 of 500 43 / 31, 8 of 120 13.8 / 9.2.  What would not leave the line's
// places 31 bits goes there too.
bool paged_few_takes(const PagedArgs& a, int max_new) {
  const long long nb = ((long long)a.max_pages * a.page_size + 15) / 16 + FSTART * FNW;
  return paged_few_rows(a, max_new) && few_units(a, few_tiles(a, max_new)) <= 0x7FFFFFFFLL / nb;
}

size_t paged_few_workspace_bytes(const PagedArgs& a, int max_new) {
  return (size_t)FMAX_WGS * FNW * (sizeof(FewJoin) + 2 * few_tiles(a, max_new) * 16 * FPR * sizeof(float));
}

hipError_t launch_paged_few(const PagedArgs& a, int e4m3, int max_new, const bf16_t* q, bf16_t* out, const void* kc, const void* vc,
                            void* workspace, hipStream_t s) {
  const long long grp = a.hpr / a.kvpr, cap = (long long)a.max_pages * a.page_size;
  const long long kb = e4m3 ? 32 : 16, nb = (cap + kb - 1) / kb;
  const int nt = few_tiles(a, max_new);
  const long long units = few_units(a, nt);
  // A cache (as wide as its table) of so few keys that a workgroup does them in the time of a second kernel's launch, while the launch
  // has one for every unit; one of so few that a wave does.  In us, 32 heads, bf16: one sequence of 300 keys 12.2 in the line, 10.8
  // a workgroup each; 128 sequences of 60 keys 29.5 in the line, 27.1 a wave each, of 120 keys 46.9 and 45.0; one sequence of 60
  // keys 9.7 a wave each, 7.9 a workgroup.  Two tiles take a workgroup's joins longer: 31 sequences of 14 keys, 32 rows each, 9.7 a
  // wave each, 12.5 a workgroup, of 120 keys 17.9 and 14.8.
  const int mode = nb <= 4 && nt > 1 ? FEW_WAVE : nb <= 8 * FNW && units <= FMAX_WGS ? FEW_WG : nb <= 8 ? FEW_WAVE : FEW_LINE;
  const int least = mode == FEW_LINE ? 2 : 1;    // both slots of a wave (one of 3001 keys, 64 / 8 heads, 1 / 2 / 4 blocks: 16.0 / 13.7 / 15.0 us)
  const long long most = mode == FEW_WG ? units * FNW : mode == FEW_WAVE ? units : units * (nb + FSTART * FNW);
  const int wgs = (int)std::min<long long>(FMAX_WGS, (most + least * FNW - 1) / (least * FNW));
  const int unit_joins = mode == FEW_LINE && units <= FMAX_WGS * FNW ? (int)units : 0;
  FewJoin* joins = reinterpret_cast<FewJoin*>(workspace);
  float* part = reinterpret_cast<float*>(joins + FMAX_WGS * FNW);
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)PHD);
  auto kernel = e4m3 ? (nt == 1 ? paged_few_kernel<true, 1> : paged_few_kernel<true, 2>)
                     : (nt == 1 ? paged_few_kernel<false, 1> : paged_few_kernel<false, 2>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(64 * FNW), 0, s, a, q, out, kc, vc, part, joins, scale_log2, least, mode, unit_joins);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || mode != FEW_LINE) return e;
  const int rows = (int)std::min<long long>(16 * nt, grp * max_new);
  hipLaunchKernelGGL(paged_few_join_kernel, dim3((unsigned)(unit_joins ? unit_joins : wgs * FNW), (unsigned)rows), dim3(64), 0, s, a, part, joins, out, 16 * nt);
  return hipGetLastError();
}

}  // namespace caat
