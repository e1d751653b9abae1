// Attention of many new tokens per sequence (prompts and chunks of them) over a paged key / value cache, gfx950.
//
// What bounds it: the two products' MFMAs and the vector work per score beside them.  A workgroup of 4 waves owns 128 consecutive
// (token, query head of the group) rows of one sequence, rank and key / value head, so grouped heads share the rows of K
// and V; a wave owns 32 of them and walks the keys in blocks of 64 with an online softmax.  (Where no sequence is said to have more
// than 64 rows, a workgroup owns 64 and two waves share 32 of them.)  Scores are computed transposed
// (S^T = K q^T, 32x32x16 MFMAs), so that a lane owns one query row and the exponentiated score registers, rounded to bf16, are the
// k-slices of the second product; V comes through the LDS transpose read.  The body is software-pipelined inside a wave: the
// score MFMAs of block b + 1 are issued one per step between the softmax arithmetic of block b.
// Probabilities are rounded to bf16, as the contiguous prompt's are, and the row sums take them so: 2^-8 of a weight at most, a relative
// error of 2.0e-3 in place of 1.6e-3 over 2048 keys, most of both the output's own rounding.  What more bits would cost (us, one value /
// two / three): 4 x 2048 tokens, 32 heads 186 / 237; 512 of 16384 in e4m3 298 / 390; 5 new tokens, 24 ragged of up to 6000 36.7 / 38.0 /
// 39.3, 24 of 6000 123 / - / 129, e4m3 86 / - / 105.
// K and V blocks (double buffered, chunk-swizzled) come from the pages directly, 16 keys of one page at a time; the table's
// entries are read two blocks ahead of their use through the scalar cache.  An e4m3 block lands as it is in a buffer of
// each wave's own and is widened to bf16 on its way into the tile, once per workgroup and not once per wave.
#include <math.h>
#include <algorithm>
#include <type_traits>
#include "caat_paged.h"

namespace caat {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef short short8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) const u32x4_t* lds_u4_t;
typedef __attribute__((address_space(3))) const char* lds_c_t;
typedef __attribute__((address_space(3))) short4_t* lds_s4_t;
typedef __attribute__((address_space(4))) const int* const_i_t;
typedef __attribute__((address_space(4))) const char* const_c_t;

static constexpr int PBK = 64;                   // keys per block
static constexpr int PCH = PHD / 8;              // 16-byte chunks per row of a tile
static constexpr int PTILE = PBK * PCH;          // chunks of a tile
static constexpr int PRAW = 4 * 256;             // chunks of the waves' e4m3 buffers: 2 KB of K and 2 KB of V each
static constexpr int PPR = PHD + 4;              // floats of a partial row: 128 sums, maximum, denominator, 2 unused
static constexpr int PWGS = 512;                 // workgroups that run at a time

// Few tiles over many keys do not fill the chip, or fill it unevenly: then the tiles of all sequences stand in one line, each as long
// as its blocks and PSTART more (its start and its results' way), and every workgroup takes an equal stretch.  In us, a tile
// per workgroup (few tiles: an equal share of its keys) / the line: 216 tiles of a ragged batch with up to 6000 keys 76 / 43, 232
// with up to 5003 90 / 82, 8 over 52000 57 / 51, 256 of one prompt over 16384 320 / 323; but 520 tiles of two prompts over 8192 keys
// 270 / 294, and 160 over 900 keys 30 / 38: the line needs PLINE_KEYS blocks of keys too.
// How even a batch is only the device knows, and its sequences' last tiles are not full; the rule looks at what the rows would fill,
// at most PLINE tiles (32 heads, 70 new tokens of up to 4000 keys, 12 even sequences 157 / 179, ragged ones 104 / 74, e4m3 107 / 61;
// 8 of 512 new tokens of up to 4096, more than PLINE when even, ragged 107 / 109, even 305 / 376).  Tiles of 64 rows, of sequences
// with few new tokens and any number of keys, take the line while its notes have room (64 / 8 heads, 5 new tokens of up to 6000 keys,
// 64 even sequences 271 / 275, ragged ones 142 / 88, e4m3 131 / 68; 256 of up to 3000 549 / 561, 192 / 174, 162 / 141; the worst, 50
// even ones, 400 tiles in 512 places, 214 / 243).
// Places count sixteenths of a block; a tile's length is taken as linear in its number, nb0 blocks the first to nb0 + slope / 16 *
// number, which is what causality makes it up to roundings.
static constexpr int PLINE = 384;
static constexpr int PLINE_ROOM = 4096;          // tiles that have a note
static constexpr int PLINE_KEYS = 24;
static constexpr int PSTART = 3 * 16;
static constexpr int PLEAST = 8 * 16;            // shortest stretch

// What the workgroup in which a tile's blocks begin says about it to the kernel that joins its parts
struct PromptJoin {
  int rows;                                      // 0: nothing to join
  int rank, kvh, first, row0;
  int begin, end, per;                           // places of the tile's blocks, length of a stretch
};

struct PromptSeq {                               // a sequence's tiles (of one rank and key / value head)
  int first, n, len, tiles, nb0, slope;
  __device__ __forceinline__ int length(int t) const { return PSTART + nb0 * 16 + slope * t; }
  __device__ __forceinline__ int before(int t) const { return t * (PSTART + nb0 * 16) + slope * (t * (t - 1) / 2); }
};

// Swizzles of the 16-byte chunks of a tile's row: K is read 32 rows x one chunk at a time, V by the transpose read, 4 rows x 64
// bytes.  Both repeat every 8 rows for V and 16 for K, which the reads' immediate offsets count on.  The e4m3 kernel writes its tiles
// 16 rows x one chunk at a time, from rows of its buffer that are swizzled for that (pr_swz).
__device__ __forceinline__ int pk_swz(int row, int c) { return c ^ (row & 15); }
template <bool E4M3> __device__ __forceinline__ int pv_swz(int row, int c) {
  return c ^ ((row & 3) << 2) ^ (E4M3 ? (row >> 2) & 1 : 0);
}
__device__ __forceinline__ int pr_swz(int row, int c) { return c ^ ((row >> 1) & 7); }
// the scores are MFMA results or -inf: a signalling input needs no quieting
__device__ __forceinline__ float pmax3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

__device__ __forceinline__ uint2 widen4(unsigned w) {   // e4m3 codes as bf16 (exact)
  return make_uint2(__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, false)),
                    __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, true)));
}
__device__ __forceinline__ uint4 widen8(const uint2& w) {
  const uint2 a = widen4(w.x), b = widen4(w.y);
  return make_uint4(a.x, a.y, b.x, b.y);
}

// LINE: the workgroup takes a stretch of the line (line_room: tiles that joins has room for), otherwise one tile
// RG: groups of 32 query rows of a tile.  4: a wave owns a group.  2: two waves share a group, each takes half of every block's keys,
// and their results meet in LDS; for sequences with at most 64 rows, of which two waves of a tile of 128 would have none (64 heads on
// 8 ranks, 8 key / value heads, 5 new tokens; tiles of 128 / 64 rows in us: 4 sequences over 6000 keys 38.7 / 33.8, e4m3 39.2 / 30.6,
// 24 over 6000 151 / 131, e4m3 118 / 92, 64 over 500 32.3 / 31.6; 8 new tokens 157 / 137 and 122 / 95 of the 24).
template <bool E4M3, bool LINE, int RG>
__global__ __launch_bounds__(256, 2) void paged_prompt_kernel(const PagedArgs a, const bf16_t* __restrict__ q, bf16_t* __restrict__ out,
                                                              const void* __restrict__ kc, const void* __restrict__ vc,
                                                              float* __restrict__ part, PromptJoin* __restrict__ joins, float scale_log2,
                                                              int line_room) {
  constexpr int ELT = E4M3 ? 1 : 2;
  constexpr int BQ = 32 * RG;                    // query rows of a tile
  constexpr int KT = RG / 2;                     // tiles of 32 keys of a block that are a wave's
  __shared__ uint4 smem[4 * PTILE + (E4M3 ? PRAW : 1)];   // K slots 0 and 1, V slots 0 and 1, 16 KB each; e4m3 buffers
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = uni(tid >> 6);
  const int rg = wave % RG, part_of = wave / RG;  // group of rows, half of the keys (0 where there is one)
  const int grp = a.hpr / a.kvpr, heads = a.T * a.kvpr;

  const int cap = a.max_pages * a.page_size;
  // blocks of keys that a tile's rows see; a token t of n sees those below len - n + t + 1
  auto tile_end = [&](int n, int len, int t) {   // may be 0 or less
    const int last_token = min(n - 1, (int)(((long long)t * BQ + BQ - 1) / grp));
    return min(min(len, cap), len - n + last_token + 1);
  };
  auto load_seq = [&](int b) {
    PromptSeq q;
    q.first = q.n = q.len = q.tiles = q.nb0 = q.slope = 0;
    if (b < a.batch) {
      q.n = seq_rows(a, b, q.first);
      q.len = max(a.lens[b], 0);
      q.tiles = (int)(((long long)q.n * grp + BQ - 1) / BQ);
      if (LINE && q.tiles > 0) {
        q.nb0 = max(1, (tile_end(q.n, q.len, 0) + PBK - 1) / PBK);
        const int nbl = max(q.nb0, (tile_end(q.n, q.len, q.tiles - 1) + PBK - 1) / PBK);
        q.slope = 16 * (nbl - q.nb0) / max(q.tiles - 1, 1);
      }
    }
    return q;
  };
  auto pick = [](const PromptSeq& q, int l) {
    return PromptSeq{__builtin_amdgcn_readlane(q.first, l), __builtin_amdgcn_readlane(q.n, l), __builtin_amdgcn_readlane(q.len, l),
                     __builtin_amdgcn_readlane(q.tiles, l), __builtin_amdgcn_readlane(q.nb0, l), __builtin_amdgcn_readlane(q.slope, l)};
  };

  // ---- which rows.  Without a line: one tile.  The launch runs through the tiles of all sequences, heads innermost
  // (a head's tiles run on one XCD, close in time, where the number of heads is a multiple of 8), a sequence's last tile,
  // which sees most keys, first.
  int b = -1, h = blockIdx.x % heads, tile = blockIdx.x / heads, base = 0, unit0 = 0, x = 0, x1 = 1, per = 1;
  PromptSeq sq = {};
  if constexpr (!LINE) {
    for (int at = 0; at < a.batch && b < 0; at += 64) {
      const PromptSeq c = load_seq(at + lane);
      const int incl = wave_sums(c.tiles);
      const unsigned long long over = __ballot(incl > tile);
      if (over) {
        const int l = __builtin_ctzll(over);
        sq = pick(c, l);
        tile = __builtin_amdgcn_readlane(incl, l) - 1 - tile;
        b = at + l;
      } else {
        tile -= __builtin_amdgcn_readlane(incl, 63);
      }
    }
    if (b < 0) return;                           // fewer tiles than the launch has room for
  } else {
    // neighbours in the line share keys: an XCD takes workgroups that stand together in it
    const int taker = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
    PromptSeq c = load_seq(lane);
    int own = c.before(c.tiles), incl = wave_sums(own), uincl = wave_sums(c.tiles);
    int total = __builtin_amdgcn_readlane(incl, 63), units = __builtin_amdgcn_readlane(uincl, 63);
    bool beyond = incl < 0;                      // a sum has passed 31 bits (one sequence cannot)
    for (int at = 64; at < a.batch; at += 64) {
      const PromptSeq d = load_seq(at + lane);
      const int sums = wave_sums(d.before(d.tiles));
      total += __builtin_amdgcn_readlane(sums, 63);
      beyond |= (sums | total) < 0;
      units += __builtin_amdgcn_readlane(wave_sums(d.tiles), 63);
    }
    // The host has checked that the line has less than 2^31 places.  A list that gives rows to many sequences can make it longer: then
    // nobody takes any.
    const bool none = __any(beyond) || (long long)total * heads > 0x7FFFFFFF;
    total = none ? 0 : total * heads;
    units = none ? 0 : units * heads;
    for (int i = units + taker * 256 + tid; i < line_room; i += gridDim.x * 256) joins[i].rows = 0;
    per = max((int)((unsigned)(total + gridDim.x - 1) / gridDim.x), PLEAST);
    x = (int)min((long long)taker * per, (long long)total);
    x1 = min(total - x, per) + x;
    if (x >= x1) return;
    for (int at = 0; at < a.batch; at += 64) {
      if (at > 0) {
        c = load_seq(at + lane);
        own = c.before(c.tiles);
        incl = wave_sums(own);
        uincl = wave_sums(c.tiles);
      }
      const unsigned long long over = __ballot(base + incl * heads > x);
      if (over) {
        const int l = __builtin_ctzll(over);
        sq = pick(c, l);
        base += __builtin_amdgcn_readlane(incl - own, l) * heads;
        unit0 += __builtin_amdgcn_readlane(uincl - c.tiles, l) * heads;
        b = at + l;
        break;
      }
      base += __builtin_amdgcn_readlane(incl, 63) * heads;
      unit0 += __builtin_amdgcn_readlane(uincl, 63) * heads;
    }
    const int one = sq.before(sq.tiles);
    h = (int)((unsigned)(x - base) / (unsigned)one);
    const int r = x - base - h * one;
    for (tile = 0; tile + 64 <= sq.tiles && sq.before(tile + 64) <= r; tile += 64) {}
    tile += __popcll(__ballot(tile + lane < sq.tiles && sq.before(tile + lane) <= r)) - 1;
  }
  const float scale0 = scale_log2;

  bool again = false;
  for (bool more = false;; more = true) {        // the tiles of the stretch
    // What a tile needs is made when it begins: what the compiler keeps from one to the next it keeps in scratch memory (32 heads, 6
    // prompts 207 us, with this 185; drafts e4m3 37.3 and 29.4).
    int lane_now = tid & 63;
    asm volatile("" : "+v"(lane_now));
    if (!LINE) asm volatile("" : "+s"(h), "+s"(tile), "+s"(b));
    const int lane = lane_now & 63, frow = lane & 31, hf = lane >> 5;
    const int n = sq.n, first = sq.first, len = sq.len;
    const int rank = h / a.kvpr, kvh = h - rank * a.kvpr;
    const int keys = min(len, cap);
    const int row0 = tile * BQ;
    const int kv_end = tile_end(n, len, tile);     // may be 0 or less
    const int all_blk = max(0, (kv_end + PBK - 1) / PBK);
    // its blocks that are this workgroup's: blk0 .. blk0 + nblk - 1
    int begin = 0, end = 1, blk0 = 0, blk1 = all_blk;
    if (LINE) {
      end = base + h * sq.before(sq.tiles) + sq.before(tile + 1);
      const int length = sq.length(tile) - PSTART;
      begin = end - length;
      if (x1 <= begin) break;                      // the stretch ends in front of the first one
      blk0 = (int)((long long)all_blk * (max(x, begin) - begin) / length);
      blk1 = (int)((long long)all_blk * (min(x1, end) - begin) / length);
    }
    const bool begins = x <= begin, all_here = begins && x1 >= end;
    const int all = blk1 - blk0;
    // Zero times a value that is not finite is NaN, also for rows that do not see its key.  A tile with such sums is begun again: its
    // blocks that every row sees as before, the other keys, at most 128 and a block's, by lanes, each for its row and dims.
    const int cut = max(0, min(all, max(min(len - n + row0 / grp + 1, keys), 0) / PBK - blk0));
    const int nblk = again ? cut : all;
    const int key0 = blk0 * PBK;
    if (more) __syncthreads();                     // everyone is done with the last tile's blocks

    // ---- Q fragments: B operand of S^T = K q^T: lane (row frow, k-half hf) holds q[16 ks + 8 hf .. + 7]
    const int qr = row0 + rg * 32 + frow;
    const int token = qr / grp, head = kvh * grp + (qr - token * grp);
    const bool row_ok = token < n;
    const long long qrow = (long long)rank * a.rows + first + token;
    const int lim = row_ok ? (int)min((long long)len - n + token + 1, (long long)keys) : kv_end;
    const int wave_lim = uni((int)min((long long)len - n + (row0 + rg * 32) / grp + 1, (long long)keys));   // of the wave's first row
    bf16x8_t qf[PHD / 16];
    const bf16_t* src = q + (row_ok ? qrow * a.ld_q + head * PHD : 0) + hf * 8;   // rows of nobody: any row, not stored
#pragma unroll
    for (int ks = 0; ks < PHD / 16; ++ks) qf[ks] = *reinterpret_cast<const bf16x8_t*>(src + ks * 16);
    scale_log2 = E4M3 && a.k_scale ? fmaxf(scale0 * a.k_scale[h], 0x1p-149f) : scale0;   // (not 0, for minus infinity's sake)

    f32x16_t oacc[PHD / 32];
#pragma unroll
    for (int t = 0; t < PHD / 32; ++t)
#pragma unroll
      for (int r = 0; r < 16; ++r) oacc[t][r] = 0.0f;
    float m_run = -INFINITY, l_run = 0.0f;         // running maximum (raw score units) and this lane's share of the row sum

    // ---- pages.  `next` holds the table's entries of the 4 groups of 16 keys of block (col, in) that is copied next; a block's
    // places are made from them when its K is copied and kept for its V, one block later.
    const const_c_t table = (const_c_t)(a.table + (long long)b * a.max_pages);
    const int gpp = a.page_size >> 4;              // groups per page
    const int n_pages = (int)a.n_pages;            // (the host has checked that it fits)
    const unsigned last_col = (unsigned)(a.max_pages - 1) * 4;
    const long long page_bytes = a.s_page * ELT, group_bytes = 16 * a.s_row * ELT;
    const bool quad = (gpp & 3) == 0;              // a block lies inside one page
    int next[4], nin;                              // entries; group inside its page behind them
    unsigned ncol;                                 // and byte offset of its column
    int pin;                                       // group inside its page of the block that is placed next (e4m3: the wave's group),
    long long pat;                                 // and its byte offset there
    {
      const int col = blk0 * 4 / gpp;
      nin = blk0 * 4 - col * gpp;
      ncol = min((unsigned)col * 4, last_col);
      pin = E4M3 ? (nin + wave) % gpp : nin;
      pat = pin * group_bytes;
    }
    const int step = 4 % gpp;
    auto fetch = [&] {
      if (quad) {
        next[0] = *(const_i_t)(table + ncol);
        if ((nin += 4) == gpp) {
          nin = 0;
          ncol = min(ncol + 4, last_col);
        }
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          next[i] = *(const_i_t)(table + ncol);
          if (++nin == gpp) {
            nin = 0;
            ncol = min(ncol + 4, last_col);
          }
        }
      }
    };
    struct Place {
      long long at[E4M3 ? 1 : 4];                  // byte offsets of the groups (e4m3: of the wave's) inside a head's pages
      unsigned have;                               // groups that have a page
    };
    auto place = [&] {
      Place p;
      if constexpr (E4M3) {
        int mine = next[0];
        if (quad) {
          p.have = (unsigned)next[0] < (unsigned)n_pages ? 15u : 0u;
        } else {
          p.have = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) p.have |= (unsigned)next[i] < (unsigned)n_pages ? 1u << i : 0u;
          mine = wave == 0 ? next[0] : wave == 1 ? next[1] : wave == 2 ? next[2] : next[3];
        }
        p.at[0] = (unsigned)mine < (unsigned)n_pages ? (unsigned)mine * page_bytes + pin * group_bytes : 0;
        pin += quad ? 4 : step;
        if (pin >= gpp) pin -= gpp;
      } else if (quad) {
        const bool ok = (unsigned)next[0] < (unsigned)n_pages;
        p.have = ok ? 15u : 0u;
        p.at[0] = ok ? (unsigned)next[0] * page_bytes + pat : 0;
#pragma unroll
        for (int i = 1; i < 4; ++i) p.at[i] = p.at[i - 1] + group_bytes;
        pat += 4 * group_bytes;
        if ((pin += 4) == gpp) {
          pin = 0;
          pat = 0;
        }
      } else {
        p.have = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const bool ok = (unsigned)next[i] < (unsigned)n_pages;
          p.at[i] = ok ? (unsigned)next[i] * page_bytes + pat : 0;
          p.have |= ok ? 1u << i : 0u;
          pat += group_bytes;
          if (++pin == gpp) {
            pin = 0;
            pat = 0;
          }
        }
      }
      return p;
    };
    const unsigned char* kh = (const unsigned char*)kc + (rank * a.s_rank + kvh * a.s_head) * ELT;
    const unsigned char* vh = (const unsigned char*)vc + (rank * a.s_rank + kvh * a.s_head) * ELT;

    // ---- global -> LDS.  bf16: a copy fills 4 rows, the wave's rows 4 wave .. + 3 of each of the 4 groups.  e4m3: a copy fills 8 rows,
    // a wave takes the group of its number, K and V.
    const unsigned row_bytes = (unsigned)(a.s_row * ELT);
    unsigned dko, dvo, dro[2] = {0, 0};
    {
      const int row = wave * 4 + (lane >> 4), phys = lane & 15;
      dko = row * row_bytes + pk_swz(row, phys) * 16;       // (the swizzles repeat every 16 rows)
      dvo = row * row_bytes + pv_swz<E4M3>(row, phys) * 16;
      if (E4M3)
        for (int i = 0; i < 2; ++i) dro[i] = (i * 8 + (lane >> 3)) * row_bytes + pr_swz(i * 8 + (lane >> 3), lane & 7) * 16;
    }
    auto issue_rows = [&](const unsigned char* base, unsigned off, const Place& p, int blk, uint4* t) {
      uint4* to = t + wave * 4 * PCH;
      const int left = kv_end - key0 - blk * PBK;  // rows from here on that anybody sees
      if (left >= PBK && p.have == 15u) {
#pragma unroll
        for (int i = 0; i < 4; ++i) dma16(make_rsrc(base + p.at[i]), off, to + i * 16 * PCH);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          dma16(make_rsrc(base + p.at[i]), (p.have >> i & 1) && i * 16 + wave * 4 + (lane >> 4) < left ? off : 0x80000000u, to + i * 16 * PCH);
      }
    };
    uint4* raw = smem + 4 * PTILE + (E4M3 ? wave * 256 : 0);
    auto issue_raw = [&](const unsigned char* base, const Place& p, int blk, uint4* t) {   // the wave's group
      const int left = p.have >> wave & 1 ? kv_end - key0 - blk * PBK - wave * 16 : 0;
      const i32x4_t rs = make_rsrc(base + p.at[0]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        dma16(rs, i * 8 + (lane >> 3) < left ? dro[i] : 0x80000000u, t + i * 64);
    };
    // the wave's group of a raw block as bf16 rows of the tile: a lane takes a quarter of a row
    auto widen = [&](const uint4* src, uint4* tile_at, bool is_v) {
      const int r = lane & 15, part = lane >> 4, row = wave * 16 + r;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const uint4 w = src[r * 8 + pr_swz(r, part * 2 + c)];
        const unsigned x[4] = {w.x, w.y, w.z, w.w};
        unsigned y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          y[2 * i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[i], 1.0f, false));
          y[2 * i + 1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[i], 1.0f, true));
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int ch = part * 4 + c * 2 + i;
          tile_at[row * PCH + (is_v ? pv_swz<E4M3>(row, ch) : pk_swz(row, ch))] = make_uint4(y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]);
        }
      }
    };
    auto kslot = [&](int blk) { return smem + (blk & 1) * PTILE; };
    auto vslot = [&](int blk) { return smem + (2 + (blk & 1)) * PTILE; };

    // Per-lane LDS addresses of the fragment reads; slot, key tile and 16-key slice go into the instructions' immediate offsets.
    //   K fragment (32 rows x one chunk): row = 32 j + frow, logical chunk 2 ks + hf
    //   V transpose read: row = 16 u + 4 hf + (i16 >> 2) (+ 8), column 32 dt + 16 half + 4 (i16 & 3)
    constexpr int TILE_BYTES = PTILE * 16;
    lds_u4_t koff[PHD / 16];
    lds_c_t voff[PHD / 32];
    {
      const lds_c_t lds0 = (lds_c_t)smem;
#pragma unroll
      for (int ks = 0; ks < PHD / 16; ++ks) koff[ks] = (lds_u4_t)(lds0 + ((part_of * 32 + frow) * PCH + pk_swz(frow, ks * 2 + hf)) * 16);
      const int i16 = lane & 15, half = (lane >> 4) & 1;
      const int vrow = 4 * hf + (i16 >> 2);
#pragma unroll
      for (int dt = 0; dt < PHD / 32; ++dt) {
        const int col = dt * 32 + half * 16 + (i16 & 3) * 4;
        voff[dt] = lds0 + (((part_of * 32 + vrow) * PCH + pv_swz<E4M3>(vrow, col >> 3)) * 16 + (col & 7) * 2);
      }
    }
    const f32x16_t zero16 = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    const bf16x2_t ones2 = {(__bf16)1.0f, (__bf16)1.0f};

    Place pk, pv;                                  // of the block whose K was copied last, of the one whose V is next
    unsigned have = 0, have_next = 0;              // groups with a page of the block in the softmax, of the one behind it

    // One key block: the scores of block blk are in `scur`; those of blk + 1 are made into `snext` under its softmax
    auto key_block = [&](int blk, f32x16_t* scur, f32x16_t* snext, auto slot_c, auto last_c) {
      constexpr int SLOT = decltype(slot_c)::value;
      constexpr bool LAST = decltype(last_c)::value;
      wait_vmcnt<0>();
      __syncthreads();                             // K(blk + 1) and V(blk) are there; everyone is done with K(blk) and V(blk - 1)
      if constexpr (E4M3) {
        // K(blk + 2) and V(blk + 1) lie in the wave's buffer, K(blk + 3) and V(blk + 2) take their place
        if (blk + 2 < nblk) widen(raw, kslot(blk), false);
        if (blk + 1 < nblk) widen(raw + 128, vslot(blk + 1), true);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        pv = pk;
        if (blk + 3 < nblk) {
          pk = place();
          fetch();
          issue_raw(kh, pk, blk + 3, raw);
        }
        if (blk + 2 < nblk) issue_raw(vh, pv, blk + 2, raw + 128);
      } else {
        pv = pk;
        if (blk + 2 < nblk) {
          pk = place();
          fetch();
          issue_rows(kh, dko, pk, blk + 2, kslot(blk));
        }
        if (blk + 1 < nblk) issue_rows(vh, dvo, pv, blk + 1, vslot(blk + 1));
      }
      const int kv0 = key0 + blk * PBK;
      // ---- mask (keys of register r: kv0 + 32 (part_of + j) + 8 (r / 4) + 4 hf + r % 4): only where some row of the wave does not see
      // the whole block, or a group has no page
      if (kv0 + PBK > wave_lim || have != 15u) {
#pragma unroll
        for (int j = 0; j < KT; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = kv0 + (part_of + j) * 32 + 8 * (r >> 2) + 4 * hf + (r & 3);
            if (key >= lim || !(have >> ((part_of + j) * 2 + (r >> 3)) & 1)) scur[j][r] = -INFINITY;
          }
      }
      have = have_next;
      have_next = E4M3 ? pv.have : pk.have;
      // ---- one MFMA per step, a scheduling fence behind each (64 keys; of 32 half as many):
      //   steps 0-15 : score MFMAs of block blk + 1 (fragments read three steps ahead); underneath: the row maximum (steps 0-3),
      //                its exchange with the other half-row (4-5), the exponentials of keys 0-31 (6-13)
      //   steps 16-31: second-product MFMAs; underneath: the exponentials of keys 32-63 (steps 16-23)
      auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
      auto kread = [&](int idx) -> u32x4_t { return koff[idx & 7][((SLOT ^ 1) * TILE_BYTES + (idx >> 3) * 32 * PCH * 16) / 16]; };
      __builtin_amdgcn_s_setprio(1);               // in front of a wave that waits for its copies (e4m3 chunk 332 -> 320 us, others even)
      float mx = -INFINITY, mxo = 0.0f, m_new = 0.0f, alpha = 1.0f, mb = 0.0f, psum = 0.0f;
      unsigned pw[8 * KT];                         // the block's probabilities, bf16 pairs
      auto prob_pair = [&](int i) {
        const int j = i >> 3, r = (i & 7) * 2;
        const float p0 = __builtin_amdgcn_exp2f(scur[j][r] * scale_log2 - mb);
        const float p1 = __builtin_amdgcn_exp2f(scur[j][r + 1] * scale_log2 - mb);
        pw[i] = pack2bf(p0, p1);
        // the row sum takes the probabilities as the second product sees them, two per instruction
        psum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pw[i]), ones2, psum, false);
        asm volatile("" : "+v"(pw[i]), "+v"(psum));   // pins the pair to this place in the stream
      };
      u32x4_t kr[3];
      if constexpr (!LAST) {
        kr[0] = kread(0);
        kr[1] = kread(1);
        kr[2] = kread(2);
      }
      fence();
#pragma unroll
      for (int idx = 0; idx < 8 * KT; ++idx) {
        if constexpr (!LAST) {
          const int j = idx >> 3, ks = idx & 7;
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, kr[idx % 3]);
          snext[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], ks == 0 ? zero16 : snext[j], 0, 0, 0);
          if (idx + 3 < 8 * KT) kr[idx % 3] = kread(idx + 3);
        }
        if (idx < 2 * KT) {
          const int j = idx >> 1, r0 = (idx & 1) * 8;
#pragma unroll
          for (int r = 0; r < 8; r += 2) mx = pmax3(mx, scur[j][r0 + r], scur[j][r0 + r + 1]);
          if (idx == 2 * KT - 1) mxo = __shfl_xor(mx, 32, 64);
        } else if (idx == 2 * KT + 1) {
          m_new = fmaxf(m_run, fmaxf(mx, mxo));
          const float mz = m_new == -INFINITY ? 0.0f : m_new;   // no key seen so far: nothing is added
          alpha = __builtin_amdgcn_exp2f((m_run - mz) * scale_log2);
          mb = mz * scale_log2;
          // prob_pair multiplies and subtracts with one rounding, and mb has a rounding of its own: half of 2^32's last place
          // makes 2^256 of a probability of 1
          if (__any(fabsf(mb) >= 0x1p24f)) {
#pragma unroll
            for (int j = 0; j < KT; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r) scur[j][r] -= mz;
            mb = 0.0f;
          }
        } else if (idx >= 2 * KT + 2 && idx < 6 * KT + 2) {
          prob_pair(idx - 2 * KT - 2);
        }
        fence();
      }
      if (__any(m_new != m_run)) {                 // the running maximum settles after the first blocks
#pragma unroll
        for (int t = 0; t < PHD / 32; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[t][r] *= alpha;
      }
      m_run = m_new;

      // ---- O^T += V^T P^T: k-slice u (16 keys): lane half hf contributes keys 16 u + 4 hf + {0 .. 3} and 16 u + 8 + 4 hf + {0 .. 3}
      auto vread = [&](int st, short4_t& v0, short4_t& v1) {
        const lds_c_t a0 = voff[st & 3] + ((2 + SLOT) * TILE_BYTES + (st >> 2) * 16 * PCH * 16);
        v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t)a0);
        v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t)(a0 + 8 * PCH * 16));
      };
      short4_t va[3], vb[3];
      vread(0, va[0], vb[0]);
      vread(1, va[1], vb[1]);
      vread(2, va[2], vb[2]);
      fence();
#pragma unroll
      for (int st = 0; st < 8 * KT; ++st) {
        const int u = st >> 2, dt = st & 3;
        const short8_t vv = {va[st % 3][0], va[st % 3][1], va[st % 3][2], va[st % 3][3],
                             vb[st % 3][0], vb[st % 3][1], vb[st % 3][2], vb[st % 3][3]};
        const bf16x8_t pfu = __builtin_bit_cast(bf16x8_t, make_uint4(pw[4 * u], pw[4 * u + 1], pw[4 * u + 2], pw[4 * u + 3]));
        oacc[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, vv), pfu, oacc[dt], 0, 0, 0);
        if (st + 3 < 8 * KT) vread(st + 3, va[st % 3], vb[st % 3]);
        if (st < 4 * KT) prob_pair(4 * KT + st);
        fence();
      }
      l_run = l_run * alpha + psum;
      __builtin_amdgcn_s_setprio(0);
    };

    if (nblk > 0) {
      // prologue: what the first iteration expects is on its way at once; the scores of block 0 wait for K(0) alone
      f32x16_t sa[KT], sb[KT];
      fetch();
      // The compiler's wait for q stands here, under the table's way and in front of the copies, which it does not know of and would
      // wait for as well
#pragma unroll
      for (int ks = 0; ks < PHD / 16; ++ks) asm volatile("" : "+v"(qf[ks]));
      pk = place();
      fetch();
      have = have_next = pk.have;
      if constexpr (E4M3) {
        uint4* k1 = vslot(1) + wave * 128;         // K(1) lands where V(1) will be widened to
        issue_raw(kh, pk, 0, raw);
        issue_raw(vh, pk, 0, raw + 128);
        if (1 < nblk) {
          pk = place();
          fetch();
          have_next = pk.have;
          issue_raw(kh, pk, 1, k1);
        }
        wait_vmcnt<0>();
        widen(raw, kslot(0), false);
        widen(raw + 128, vslot(0), true);
        if (1 < nblk) widen(k1, kslot(1), false);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (1 < nblk) issue_raw(vh, pk, 1, raw + 128);   // V(1) stays in the buffer for the first iteration
        if (2 < nblk) {
          pk = place();
          fetch();
          issue_raw(kh, pk, 2, raw);
        }
      } else {
        issue_rows(kh, dko, pk, 0, kslot(0));
        issue_rows(vh, dvo, pk, 0, vslot(0));
        if (1 < nblk) {
          pk = place();
          fetch();
          have_next = pk.have;
          issue_rows(kh, dko, pk, 1, kslot(1));
          wait_vmcnt<8>();
        } else {
          wait_vmcnt<4>();
        }
      }
      __syncthreads();
#pragma unroll
      for (int j = 0; j < KT; ++j)
#pragma unroll
        for (int ks = 0; ks < PHD / 16; ++ks) {
          const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, koff[ks][(j * 32 * PCH * 16) / 16]);
          sa[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[ks], ks == 0 ? zero16 : sa[j], 0, 0, 0);
        }
      int blk = 0;
      for (; blk + 2 < nblk; blk += 2) {
        key_block(blk, sa, sb, std::integral_constant<int, 0>{}, std::false_type{});
        key_block(blk + 1, sb, sa, std::integral_constant<int, 1>{}, std::false_type{});
      }
      if (blk + 1 < nblk) {
        key_block(blk, sa, sb, std::integral_constant<int, 0>{}, std::false_type{});
        key_block(blk + 1, sb, sa, std::integral_constant<int, 1>{}, std::true_type{});
      } else {
        key_block(blk, sa, sb, std::integral_constant<int, 0>{}, std::true_type{});
      }
    }

    if (again) {
      for (int kk = cut * PBK; kk < all * PBK; ++kk) {
        const int key = key0 + kk;
        if (key >= kv_end) break;
        if (RG == 2 && (kk >> 5 & 1) != part_of) continue;
        const int col = key / a.page_size, page = *(const_i_t)(table + col * 4);
        if ((unsigned)page >= (unsigned)n_pages) continue;
        const long long at = page * page_bytes + (key - col * a.page_size) * (long long)row_bytes;
        float s = 0.0f;
#pragma unroll
        for (int ks = 0; ks < PHD / 16; ++ks) {
          uint4 w;
          if constexpr (E4M3) w = widen8(*reinterpret_cast<const uint2*>(kh + at + ks * 16 + hf * 8));
          else w = *reinterpret_cast<const uint4*>(kh + at + (ks * 16 + hf * 8) * 2);
          s += dot8(w, *reinterpret_cast<const uint4*>(src + ks * 16));
        }
        s += __shfl_xor(s, 32, 64);
        if (key >= lim) continue;
        const float m_new = fmaxf(m_run, s), mz = m_new == -INFINITY ? 0.0f : m_new;
        const float alpha = __builtin_amdgcn_exp2f((m_run - mz) * scale_log2);
        const float p = lo_bf(pack2bf(__builtin_amdgcn_exp2f((s - mz) * scale_log2), 0.0f));
        m_run = m_new;
        l_run = l_run * alpha + (hf == 0 ? p : 0.0f);
#pragma unroll
        for (int dt = 0; dt < PHD / 32; ++dt)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int d = dt * 32 + k * 8 + hf * 4;
            uint2 w;
            if constexpr (E4M3) w = widen4(*reinterpret_cast<const unsigned*>(vh + at + d));
            else w = *reinterpret_cast<const uint2*>(vh + at + d * 2);
            const float v[4] = {lo_bf(w.x), hi_bf(w.x), lo_bf(w.y), hi_bf(w.y)};
#pragma unroll
            for (int r = 0; r < 4; ++r) oacc[dt][4 * k + r] = oacc[dt][4 * k + r] * alpha + p * v[r];
          }
      }
    } else if (cut < all) {
      float odd = 0.0f;                            // NaN where a sum is not finite
#pragma unroll
      for (int t = 0; t < PHD / 32; ++t)
#pragma unroll
        for (int r = 0; r < 16; ++r) odd = __builtin_fmaf(oacc[t][r], 0.0f, odd);
      const bool wave_odd = __any(odd != odd);
      int* said = reinterpret_cast<int*>(smem + 4 * PTILE);   // (e4m3: a wave's own buffer, which has been read)
      constexpr int NEXT = E4M3 ? 256 * 4 : 1;
      if (lane == 0) said[wave * NEXT] = wave_odd;
      __syncthreads();
      if (said[0] | said[NEXT] | said[2 * NEXT] | said[3 * NEXT]) {
        again = true;
        continue;
      }
    }
    again = false;

    // ---- normalise and store: lane holds out[row][32 dt + 8 (r / 4) + 4 hf + r % 4]
    l_run += __shfl_xor(l_run, 32, 64);
    if constexpr (RG == 2) {
      // the second halves' results through the tiles' place: 16 chunks of 4 sums per lane, then maximum and denominator
      float4* po = reinterpret_cast<float4*>(smem) + rg * 16 * 64;
      float2* pm = reinterpret_cast<float2*>(reinterpret_cast<float4*>(smem) + 2 * 16 * 64) + rg * 64;
      __syncthreads();
      if (part_of == 1) {
#pragma unroll
        for (int c = 0; c < 16; ++c)
          po[c * 64 + lane] = make_float4(oacc[c >> 2][(c & 3) * 4], oacc[c >> 2][(c & 3) * 4 + 1], oacc[c >> 2][(c & 3) * 4 + 2],
                                          oacc[c >> 2][(c & 3) * 4 + 3]);
        pm[lane] = make_float2(m_run, l_run);
      }
      __syncthreads();
      if (part_of == 0) {
        const float2 ml = pm[lane];
        const float m_new = fmaxf(m_run, ml.x), mz = m_new == -INFINITY ? 0.0f : m_new;
        const float f0 = __builtin_amdgcn_exp2f((m_run - mz) * scale_log2), f1 = __builtin_amdgcn_exp2f((ml.x - mz) * scale_log2);
        m_run = m_new;
        l_run = l_run * f0 + ml.y * f1;
#pragma unroll
        for (int c = 0; c < 16; ++c) {
          const float4 o = po[c * 64 + lane];
          const float v[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) oacc[c >> 2][(c & 3) * 4 + k] = oacc[c >> 2][(c & 3) * 4 + k] * f0 + v[k] * f1;
        }
      }
    }
    const bool stores = row_ok && part_of == 0;
    if (LINE && begins && tid == 0) {
      PromptJoin* j = joins + unit0 + h * sq.tiles + tile;
      if ((unsigned)(unit0 + h * sq.tiles + tile) < (unsigned)line_room)
        *j = PromptJoin{all_here ? 0 : min(BQ, n * grp - row0), rank, kvh, first, row0, begin, end, per};
    }
    if (LINE && !all_here) {
      const int taker = blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
      if (stores) {
        float* o = part + ((2LL * taker + (begins ? 1 : 0)) * BQ + rg * 32 + frow) * PPR;
#pragma unroll
        for (int dt = 0; dt < PHD / 32; ++dt)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *reinterpret_cast<float4*>(o + dt * 32 + k * 8 + hf * 4) =
                make_float4(oacc[dt][k * 4], oacc[dt][k * 4 + 1], oacc[dt][k * 4 + 2], oacc[dt][k * 4 + 3]);
        if (hf == 0) *reinterpret_cast<float2*>(o + PHD) = make_float2(m_run * scale_log2, l_run);
      }
    } else if (stores) {
      float inv = (E4M3 && a.v_scale ? a.v_scale[h] : 1.0f) / l_run;
      if (l_run == 0.0f) {                         // no key seen, or all scores minus infinity: zeros, whatever the values hold
        inv = 0.0f;
#pragma unroll
        for (int t = 0; t < PHD / 32; ++t)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[t][r] = 0.0f;
      }
      bf16_t* o = out + (qrow * a.hpr + head) * PHD;
#pragma unroll
      for (int dt = 0; dt < PHD / 32; ++dt)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint2 w;
          w.x = pack2bf(oacc[dt][k * 4 + 0] * inv, oacc[dt][k * 4 + 1] * inv);
          w.y = pack2bf(oacc[dt][k * 4 + 2] * inv, oacc[dt][k * 4 + 3] * inv);
          *reinterpret_cast<uint2*>(o + dt * 32 + k * 8 + hf * 4) = w;
        }
    }
    // ---- the next tile
    if (!LINE || x1 <= end) break;
    x = end;
    if (++tile == sq.tiles) {
      tile = 0;
      if (++h == heads) {
        h = 0;
        base += heads * sq.before(sq.tiles);
        unit0 += heads * sq.tiles;
        do {
          if (++b >= a.batch) return;
          sq = load_seq(b);                        // (all lanes the same)
          sq = pick(sq, 0);
        } while (sq.tiles == 0);
      }
    }
  }
}

// Joins the parts of a tile, in the order of the keys: 32 threads, 4 channels each, for a row and every SUBS-th part of it.
template <int SUBS>
__global__ __launch_bounds__(256) void paged_prompt_join_kernel(const PagedArgs a, const float* __restrict__ part,
                                                                const PromptJoin* __restrict__ joins, bf16_t* __restrict__ out, int bq) {
  __shared__ float4 s_num[SUBS > 1 ? 256 : 1];
  __shared__ float2 s_ml[SUBS];
  const PromptJoin j = joins[blockIdx.x];
  const int sub = (threadIdx.x >> 5) % SUBS, r = blockIdx.y * (8 / SUBS) + (threadIdx.x >> 5) / SUBS, c = (threadIdx.x & 31) * 4;
  if (r >= j.rows) return;                       // (SUBS 8: the whole workgroup)
  const int w0 = j.begin / j.per, parts = (j.end - 1) / j.per + 1 - w0;
  float M = -INFINITY, den = 0.0f;
  float4 num = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int p0 = sub; p0 < parts; p0 += 4 * SUBS) {
    float2 ml[4];
    float4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int k = min(p0 + i * SUBS, parts - 1);
      const float* q = part + ((2LL * (w0 + k) + (k == 0 ? 1 : 0)) * bq + r) * PPR;   // the first one's lies behind that of the tile before
      ml[i] = *reinterpret_cast<const float2*>(q + PHD);
      v[i] = *reinterpret_cast<const float4*>(q + c);
      if (p0 + i * SUBS >= parts) ml[i].x = -INFINITY;
    }
    const float m_new = fmaxf(fmaxf(M, ml[0].x), fmaxf(fmaxf(ml[1].x, ml[2].x), ml[3].x)), mb = m_new == -INFINITY ? 0.0f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(M - mb);
    M = m_new;
    den *= alpha;
    num = make_float4(num.x * alpha, num.y * alpha, num.z * alpha, num.w * alpha);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p0 + i * SUBS >= parts) break;
      const float f = __builtin_amdgcn_exp2f(ml[i].x - mb);
      den += ml[i].y * f;
      num = make_float4(num.x + v[i].x * f, num.y + v[i].y * f, num.z + v[i].z * f, num.w + v[i].w * f);
    }
  }
  if constexpr (SUBS > 1) {
    s_num[threadIdx.x] = num;
    if ((threadIdx.x & 31) == 0) s_ml[sub] = make_float2(M, den);
    __syncthreads();
    if (threadIdx.x >= 32) return;
    M = s_ml[0].x;
#pragma unroll
    for (int k = 1; k < SUBS; ++k) M = fmaxf(M, s_ml[k].x);
    const float mb = M == -INFINITY ? 0.0f : M;
    den = 0.0f;
    num = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < SUBS; ++k) {
      const float f = __builtin_amdgcn_exp2f(s_ml[k].x - mb);
      const float4 v = s_num[k * 32 + threadIdx.x];
      den += s_ml[k].y * f;
      num = make_float4(num.x + v.x * f, num.y + v.y * f, num.z + v.z * f, num.w + v.w * f);
    }
  }
  const int grp = a.hpr / a.kvpr, qr = j.row0 + r, token = qr / grp, h = j.kvh * grp + (qr - token * grp);
  const float inv = den == 0.0f ? 0.0f : (a.v_scale ? a.v_scale[j.rank * a.kvpr + j.kvh] : 1.0f) / den;
  if (den == 0.0f) num = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  *reinterpret_cast<uint2*>(out + (((long long)j.rank * a.rows + j.first + token) * a.hpr + h) * PHD + c) =
      make_uint2(pack2bf(num.x * inv, num.y * inv), pack2bf(num.z * inv, num.w * inv));
}

// query rows of a tile.  (max_new is the caller's word; more tokens than that only make more tiles.)
static int prompt_rows(const PagedArgs& a, int max_new) { return (long long)max_new * (a.hpr / a.kvpr) <= 64 ? 64 : 128; }

// at most as many tiles (of all heads) as this: a sequence's last one is not full
static long long prompt_tiles(const PagedArgs& a, int bq) {
  const long long rows = (long long)a.rows * (a.hpr / a.kvpr);
  return std::min((rows + bq - 1) / bq + a.batch - 1, rows) * a.T * a.kvpr;
}

// as many as the line may have, 0: no line
static int prompt_line(const PagedArgs& a, int bq) {
  const long long tiles = prompt_tiles(a, bq), full = ((long long)a.rows * (a.hpr / a.kvpr) + bq - 1) / bq * a.T * a.kvpr;
  return tiles <= PLINE_ROOM && (bq == 64 || full <= PLINE) ? (int)tiles : 0;
}

size_t paged_prompt_workspace_bytes(const PagedArgs& a, int max_new) {
  return PLINE_ROOM * sizeof(PromptJoin) + 2 * PWGS * (size_t)(prompt_rows(a, max_new) * PPR) * sizeof(float);   // of the line
}

template <int RG>
static auto prompt_kernel(int e4m3, int line) {
  return e4m3 ? (line ? paged_prompt_kernel<true, true, RG> : paged_prompt_kernel<true, false, RG>)
              : (line ? paged_prompt_kernel<false, true, RG> : paged_prompt_kernel<false, false, RG>);
}

hipError_t launch_paged_prompt(const PagedArgs& a, int e4m3, int max_new, const bf16_t* q, bf16_t* out, const void* kc, const void* vc,
                               void* workspace, hipStream_t s) {
  const int bq = prompt_rows(a, max_new);
  const long long tiles = prompt_tiles(a, bq), most = ((long long)a.max_pages * a.page_size / PBK + 2) * 16 + PSTART;   // of a tile
  const int line_room = most >= PLINE_KEYS * 16 && most <= 0x7FFFFFFFLL / tiles ? prompt_line(a, bq) : 0;
  PromptJoin* joins = reinterpret_cast<PromptJoin*>(workspace);
  float* part = reinterpret_cast<float*>(joins + PLINE_ROOM);
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)PHD);
  auto kernel = bq == 64 ? prompt_kernel<2>(e4m3, line_room) : prompt_kernel<4>(e4m3, line_room);
  const long long wgs = line_room ? std::min<long long>(PWGS, (most * tiles / PLEAST + 8) / 8 * 8) : tiles;
  hipLaunchKernelGGL(kernel, dim3((unsigned)wgs), dim3(256), 0, s, a, q, out, kc, vc, part, joins, scale_log2, line_room);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !line_room) return e;
  if (tiles <= PWGS / 8)                         // many parts of a tile (8 tiles over 52000 keys 82 -> 66 us, 64 over 16384: 79 and 78)
    hipLaunchKernelGGL(paged_prompt_join_kernel<8>, dim3((unsigned)tiles, (unsigned)bq), dim3(256), 0, s, a, part, joins, out, bq);
  else
    hipLaunchKernelGGL(paged_prompt_join_kernel<1>, dim3((unsigned)tiles, (unsigned)(bq / 8)), dim3(256), 0, s, a, part, joins, out, bq);
  return hipGetLastError();
}

}  // namespace caat
