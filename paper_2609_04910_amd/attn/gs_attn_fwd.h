// gs_attn_fwd.h -- softmax attention, forward:
//   out_m = sum_n w_mn v_n / sum_n w_mn ,  w_mn = exp(scale q_m.k_n) ,
//   lse_m = log sum_n w_mn ,
// over the keys n that row m sees, in one pass: the weights are taken relative to
// a running offset o_m of the exponent (log2 units), and where a row's largest
// exponent outgrows it the sums so far are scaled by exp2(old - new).
//
// k_attn_fwd: a workgroup of NW waves streams 64-key (DP = 256: 32-key) tiles of K
// and V through an LDS ring, one barrier a tile; wave w owns 16*NQ rows whose query
// operands and output sums stay in registers.  Bound by the matrix cores: 16384
// tokens, 16 query and 4 key heads, D = 128, causal 982 us, 1.12 PFLOP/s (a library
// product of 8192 cubed: 1.28).
// k_attn_rows: the same for few rows, bound by reading K and V: one token of 64
// sequences of 4096 keys, 8 key heads, D = 128 208 us, 5.2 TB/s (a streaming read:
// 5.6).
// Both can work on a part of a row's keys; k_attn_join then joins the parts.
#pragma once

#include "gs_attn.h"

namespace gs {

// Where a row's keys lie: rows of an array (dense and packed), or pages.
struct AttnPages {
  const int32_t* table;    // B x width page numbers; NULL: not paged
  const int32_t* lens;     // keys of each sequence, new ones included
  int64_t page_stride_k, page_stride_v;  // bytes
  int32_t width, pages, size;
  int32_t shift;           // log2 of size where it is a power of two, else -1
};

struct AttnFwdArgs {
  AttnShape s;
  AttnArray q, k, v, out;
  AttnArray low;           // out - rounded; p NULL: not wanted
  float* lse;              // NULL: not wanted
  int64_t lse_sb, lse_sh;  // elements
  AttnPages pg;
  int32_t per;             // rows that a token takes: 1, or G where a key head's query heads are packed
  int32_t tiles;           // dense: row tiles of a sequence; packed: tile slots
  int32_t heads;           // heads of the grid, all sequences of a dense call together
  int32_t neg;             // scale < 0: queries enter negated
  float c;                 // |scale| log2 e
  int32_t wgs;             // workgroups of one part
  int32_t splits;          // parts that a row's keys are cut into (1: results are written at once)
  float* part_o;           // splits x rows x query heads x C: sums of weights times values
  float* part_z;           // splits x rows x query heads x 2: offset (or kNoKeys) and sum of weights
};

// Weights lie below 2^15 relative to the offset, the largest of a row between
// 2^7 and 2^15: fp16 then holds weights down to 2^-21 of the largest in full
// precision, and the sums are scaled again only where the largest exponent grows
// by more than 8.
constexpr float kOffsetBelow = 7.0f;
constexpr float kOffsetLimit = 15.0f;
constexpr float kNoOffset = -3.0e38f;
// The offset that a row starts with, and keeps, where it sees no key.  (One whose
// scores are all -inf keeps kNoOffset: it is no empty row, and its result is 0 / 0.)
constexpr float kNoKeys = -3.2e38f;

__device__ __forceinline__ int page_index(const AttnPages& pg, int j) {
  return pg.shift >= 0 ? j >> pg.shift : (int)((uint32_t)j / (uint32_t)pg.size);
}
__device__ __forceinline__ const char* page_row(const AttnPages& pg, const char* base, int64_t page_stride, int64_t sr,
                                                int page, int j) {
  const int off = pg.shift >= 0 ? j & (pg.size - 1) : (int)((uint32_t)j % (uint32_t)pg.size);
  return base + page * page_stride + off * sr;
}

// The part of a sequence's page table that a stretch of keys needs, in LDS: waiting
// for a page number from memory between a tile's copies would wait for the copies
// too.  Numbers outside the cache become -1, and their rows are read from page 0
// (the scores of such keys are set to NaN).
constexpr int kSlice = 2048;  // page numbers; a stretch is at most kSlice - 2 pages long
struct PageSlice {
  const int32_t* e;
  int first;
  bool bad;  // whether a number lies outside the cache
  // Keys [key0, key1) of sequence b; a barrier of the workgroup.
  __device__ __forceinline__ void load(const AttnPages& pg, int32_t* lds, int b, int key0, int key1, int threads) {
    e = lds;
    first = page_index(pg, key0);
    const int n = page_index(pg, key1 - 1) - first + 1;
    bool out = false;
    for (int i = threadIdx.x; i < n; i += threads) {
      const int p = pg.table[(int64_t)b * pg.width + first + i];
      const bool ok = (uint32_t)p < (uint32_t)pg.pages;
      lds[i] = ok ? p : -1;
      out |= !ok;
    }
    bad = __syncthreads_or(out);
  }
  __device__ __forceinline__ int number(const AttnPages& pg, int j) const { return e[page_index(pg, j) - first]; }
};

// Keys (rows) of a streamed tile: two stages of K and V take 64 KiB, so two
// workgroups share a CU.  (32-key tiles in three or four stages: 4 - 10 % slower.)
template <int DP>
constexpr int attn_keys() { return DP == 256 ? 32 : 64; }

// Query operand: columns 32c + 8g .. +7 of one row, zero past the width.
template <typename T>
__device__ __forceinline__ uint4 column_operand(const char* row, int vec, int width, int c, int flip) {
  const int e0 = 32 * c + 8 * ((threadIdx.x & 63) >> 4);
  uint4 x{0, 0, 0, 0};
  if (vec) {
    if (e0 < width) x = *reinterpret_cast<const uint4*>(row + e0 * 2);
  } else {
    uint32_t y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = e0 + e < width ? reinterpret_cast<const uint16_t*>(row)[e0 + e] : 0u;
    x = uint4{y[0] | y[1] << 16, y[2] | y[3] << 16, y[4] | y[5] << 16, y[6] | y[7] << 16};
  }
  if (flip) x.x ^= 0x80008000u, x.y ^= 0x80008000u, x.z ^= 0x80008000u, x.w ^= 0x80008000u;
  return x;
}

// Copies a tile of keys and values key0 .. from the pages; rows past key end - 1 are
// others of the cache (they are masked, and cleaned).  Where a page holds a power
// of two of at least 8 rows, the rows of a wave's copy lie in one page: its
// address is then found once a copy, in scalar registers.
template <bool WIDE, typename Copy>
__device__ __forceinline__ void copy_pages(const AttnFwdArgs& a, const PageSlice& pages, const Copy& tc, char* kt,
                                           char* vt, const char* kb, const char* vb, int key0, int end) {
  const AttnPages& pg = a.pg;
  if (WIDE && pg.shift >= 3) {
    int page[Copy::N], off[Copy::N];
#pragma unroll
    for (int i = 0; i < Copy::N; ++i) {
      const int j = min(key0 + tc.wave_row() + i * Copy::STEP, (end - 1) & ~(Copy::RW - 1));
      page[i] = pages.number(pg, j);
      off[i] = j & (pg.size - 1);
    }
#pragma unroll
    for (int i = 0; i < Copy::N; ++i) page[i] = max(uniform(page[i]), 0);
    tc.wide_bases(kt, a.s.D, (uint32_t)a.k.sr, [&](int i) { return kb + page[i] * pg.page_stride_k + off[i] * a.k.sr; });
    tc.wide_bases(vt, a.s.C, (uint32_t)a.v.sr, [&](int i) { return vb + page[i] * pg.page_stride_v + off[i] * a.v.sr; });
    return;
  }
  auto key_of = [&](int i) { return min(key0 + tc.row0 + i * Copy::STEP, end - 1); };
  auto page = [&](int i) { return max(pages.number(pg, key_of(i)), 0); };
  auto krow = [&](int i) { return page_row(pg, kb, pg.page_stride_k, a.k.sr, page(i), key_of(i)); };
  auto vrow = [&](int i) { return page_row(pg, vb, pg.page_stride_v, a.v.sr, page(i), key_of(i)); };
  if (WIDE) {
    tc.wide_rows(kt, a.s.D, krow);
    tc.wide_rows(vt, a.s.C, vrow);
  } else {
    tc.narrow_rows(kt, a.s.D, krow);
    tc.narrow_rows(vt, a.s.C, vrow);
  }
}

// Sets the bits of the lane's results that infinities among the values of a tile
// reach: +inf in the first NB words of each column tile, -inf in the next, NaN in
// both (inf - inf is NaN).  The values are read from the caller's array again;
// products of indicators tell which columns see a row that has one.
template <typename T, int DP, int BK, int NQ, bool PAGED, int NB2>
__device__ __forceinline__ void found_infinities(const AttnFwdArgs& a, const char* vb, int b, int kn, int key0,
                                              const int (&lo)[NQ], const int (&hi)[NQ], uint32_t (&bits)[NB2],
                                              bool first) {
  constexpr uint32_t e = exponent_bits<T>(), one = __is_same(T, F16) ? 0x3c00u : 0x3f80u;
  constexpr int NB = NB2 / (2 * NQ);
  const int lane = threadIdx.x & 63, g = lane >> 4;
  if (first)
    for (int i = 0; i < NB2; ++i) bits[i] = 0;
#pragma nounroll
  for (int h = 0; h < BK / 32; ++h) {
#pragma nounroll
    for (int ct = 0; ct < (a.s.C + 15) / 16; ++ct) {
      uint32_t u[8], d[8];
#pragma unroll
      for (int z = 0; z < 8; ++z) {
        const int j = min(key0 + 32 * h + 16 * (z >> 2) + 4 * g + (z & 3), kn - 1), c = 16 * ct + (lane & 15);
        const char* p;
        if (PAGED) {
          const int page = a.pg.table[(int64_t)b * a.pg.width + page_index(a.pg, j)];
          p = page_row(a.pg, vb, a.pg.page_stride_v, a.v.sr, (uint32_t)page < (uint32_t)a.pg.pages ? page : 0, j);
        } else {
          p = vb + (int64_t)j * a.v.sr;
        }
        const uint32_t x = c < a.s.C ? reinterpret_cast<const uint16_t*>(p)[c] : 0u;
        u[z] = (x & e) == e && x != (e | 0x8000u) ? one : 0u;
        d[z] = (x & e) == e && x != e ? one : 0u;
      }
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        uint32_t w[8];
#pragma unroll
        for (int z = 0; z < 8; ++z) {
          const int j = key0 + 32 * h + 16 * (z >> 2) + 4 * g + (z & 3);
          w[z] = j >= lo[n] && j < hi[n] ? one : 0u;
        }
        const auto pack = [](const uint32_t(&x)[8]) {
          return uint4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
        };
        const floatx4 pu = mfma_qk<T>(pack(u), pack(w), floatx4{0, 0, 0, 0});
        const floatx4 pd = mfma_qk<T>(pack(d), pack(w), floatx4{0, 0, 0, 0});
        uint32_t mu = 0, md = 0;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (pu[r] > 0.0f) mu |= 1u << r;
          if (pd[r] > 0.0f) md |= 1u << r;
        }
        bits[(2 * n) * NB + ct / 8] |= mu << (4 * (ct & 7));
        bits[(2 * n + 1) * NB + ct / 8] |= md << (4 * (ct & 7));
      }
    }
  }
}

// Adds to the sums of column tile n, rows 4 ct .. of the lane's results, the
// infinities that reach them.
template <int NB, int NB2>
__device__ __forceinline__ void add_infinities(const uint32_t (&bits)[NB2], int n, int ct, floatx4& y) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t bit = 1u << ((4 * ct + e) & 31);
    if (bits[2 * n * NB + ct / 8] & bit) y[e] += __builtin_inff();
    if (bits[(2 * n + 1) * NB + ct / 8] & bit) y[e] -= __builtin_inff();
  }
}

// What a workgroup works on: a tile of rows of one sequence and key head, and a
// stretch of its keys.
struct AttnJob {
  int b, kvh, head;    // head: the first of the `per` query heads of the rows, over per
  AttnSeq sq;
  int ahead;           // place of the first query among the keys (causal)
  int rows, limit;     // rows of the sequence (token-major, then its query heads), and rows that the call owns
  int r0;              // first row of the tile
  int part;            // which split
};

// The sequence with the rank-th longest of B lengths, so that a batch's long
// sequences start first and its short ones fill in: 64 sequences of 2048 to 8192
// keys, 8 key heads 333 -> 278 us (5.1 TB/s; equal lengths of 4096 205 -> 211 us).
// More sequences than lanes even out by their number.
__device__ __forceinline__ int by_length(const int32_t* lens, int B, int rank) {
  if (B > 64) return rank;
  const int lane = threadIdx.x & 63;
  const int place = place_by(lane < B ? lens[lane] : 0, B);
  return __builtin_ctzll(__ballot(lane < B && place == rank));
}

// Returns whether there is anything to do (rows of no sequence are handled here).
// FOLD: two workgroups share a CU.  Not so for few rows, where no two workgroups
// share keys either: there (paged) the sequences of most keys come first.
template <int ROWS, bool PAGED, bool FOLD>
__device__ __forceinline__ bool attn_job(const AttnFwdArgs& a, AttnJob& w) {
  const AttnShape& s = a.s;
  int id = FOLD ? folded(blockIdx.x, gridDim.x) : blockIdx.x;
  w.part = 0;
  if (a.splits > 1) {
    // all first parts, then all second ones, ...: parts without keys then fall on
    // every XCD alike
    w.part = id / a.wgs;
    id -= w.part * a.wgs;
  }
  int tile, head;
  block_place(id, a.heads, tile, head);
  if (s.packed) {
    const int slot = tile;
    int n;
    w.b = packed_tile(s.q_index, s.B, s.M, a.per, ROWS, slot, PAGED ? a.pg.lens : nullptr, tile, n);
    if (w.b == kNoRow) {  // slots past the last tile: rows of no sequence
      if (s.zero_rest && w.part == 0) {
        const int part = slot - tile, parts = a.tiles - tile;
        const RestRows rest(s.q_index, s.B, s.M);
        for (int h = head * a.per; h < (head + 1) * a.per; ++h) {
          if (s.zero_rest & kRestOut) {
            zero_rest_rows(a.out, h, s.C, rest, part, parts);
            if (a.low.p) zero_rest_rows(a.low, h, s.C, rest, part, parts);
          }
          if (a.lse && (s.zero_rest & kRestLse))
            for (int64_t i = part + (int64_t)threadIdx.x * parts; i < rest.n; i += (int64_t)blockDim.x * parts)
              a.lse[h * a.lse_sh + rest.row((int)i)] = -__builtin_inff();
        }
      }
      return false;
    }
    tile = n - 1 - tile;  // the tiles that see most keys first
  } else {
    const int per_seq = a.heads / s.B;
    if (PAGED && !FOLD) {
      const int p = id % a.heads;
      w.b = by_length(a.pg.lens, s.B, p / per_seq);
      head = p % per_seq;
    } else {
      w.b = head / per_seq;
      head -= w.b * per_seq;
    }
    tile = a.tiles - 1 - tile;  // the tiles that see most keys first
  }
  w.head = head;
  w.kvh = a.per > 1 ? head : head / s.G;
  if (PAGED) {
    if (s.packed)
      seq_side(s.q_index, 1, w.b, s.M, w.sq.q0, w.sq.qn);
    else
      w.sq.q0 = 0, w.sq.qn = s.M;
    w.sq.q0 = uniform(w.sq.q0), w.sq.qn = uniform(w.sq.qn);
    w.sq.k0 = 0;
    // a cache without pages holds no keys; where a sequence is longer than its table
    // has room for, its tokens keep their places and the keys end with the table
    const int64_t room = a.pg.pages > 0 ? (int64_t)a.pg.width * a.pg.size : 0;
    const int len = uniform(max(a.pg.lens[w.b], 0));
    w.sq.kn = min(len, (int)min(room, (int64_t)0x3fffffff));
    w.ahead = len - w.sq.qn;
  } else {
    w.sq = seq_of(s, w.b);
    w.ahead = w.sq.kn - w.sq.qn;
  }
  w.rows = w.sq.qn * a.per;
  w.limit = s.packed ? w.rows : s.M * a.per;
  w.r0 = tile * ROWS;
  return w.r0 < w.limit;
}

// Keys that the rows [first, last] see: all of [in_lo, in_hi), none outside [lo, hi).
struct KeyRange {
  int lo = 0, hi = 0, in_lo = 0, in_hi = 0;
};
__device__ __forceinline__ KeyRange keys_of_rows(const AttnFwdArgs& a, const AttnJob& w, int first, int last) {
  KeyRange r;
  if (first >= w.rows) return r;
  query_range(a.s, first / a.per, w.ahead, w.sq.kn, r.lo, r.in_hi);
  query_range(a.s, min(last, w.rows - 1) / a.per, w.ahead, w.sq.kn, r.in_lo, r.hi);
  return r;
}

// This workgroup's part of the keys [lo, hi): whole tiles, no part shorter than
// kLeastPart keys.
constexpr int kLeastPart = 256;
__device__ __forceinline__ void split_keys(const AttnFwdArgs& a, const AttnJob& w, int tile, int& lo, int& hi) {
  lo = lo / tile * tile;
  if (a.splits == 1) return;
  int each = max(kLeastPart, (hi - lo + a.splits - 1) / a.splits);
  each = (each + tile - 1) / tile * tile;
  const int64_t first = lo + (int64_t)w.part * each;
  hi = first < hi ? (int)min(first + each, (int64_t)hi) : lo;
  lo = first < hi ? (int)first : lo;
}

// A wave's rows: NQ tiles of 16, row 16 n + l%16 in the lane's column of tile n.
template <typename T, int DP, int NQ>
struct AttnRows {
  static constexpr int NC = DP / 32, NO = DP / 16;
  int lo[NQ], hi[NQ];      // keys that the row sees
  uint4 q[NQ][NC];
  floatx4 o[NO][NQ];       // sums of weights times values
  float off[NQ], sum[NQ];  // offset of the exponents (start_offsets), sum of the weights in this lane

  // Rows wr0 ..; rows past the end repeat the last one (nothing of them is written).
  __device__ __forceinline__ void start(const AttnFwdArgs& a, const AttnJob& w, int wr0) {
    const int col = threadIdx.x & 15;
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const int r = min(wr0 + 16 * n + col, w.rows - 1);
      const int token = a.per > 1 ? r / a.per : r;
      const int h = a.per > 1 ? w.head * a.per + (r - token * a.per) : w.head;
      lo[n] = hi[n] = 0;
      sum[n] = 0.0f;
#pragma unroll
      for (int ct = 0; ct < NO; ++ct) o[ct][n] = floatx4{0, 0, 0, 0};
      if (w.rows > 0) {
        query_range(a.s, token, w.ahead, w.sq.kn, lo[n], hi[n]);
        const char* p = a.q.p + w.b * a.q.sb + (int64_t)(w.sq.q0 + token) * a.q.sr + h * a.q.sh;
#pragma unroll
        for (int c = 0; c < NC; ++c) q[n][c] = column_operand<T>(p, a.q.vec, a.s.D, c, a.neg);
      }
    }
  }

  // Where the offsets start: the keys of this workgroup are [from, to).
  __device__ __forceinline__ void start_offsets(int from, int to) {
#pragma unroll
    for (int n = 0; n < NQ; ++n) off[n] = max(lo[n], from) < min(hi[n], to) ? kNoOffset : kNoKeys;
  }

  // The keys key0 .. of a tile, H steps of 32.  masked: some row does not see all
  // of them; pages->bad: some of them may lie on a page outside the cache.
  template <int H>
  __device__ __forceinline__ void attend(const AttnFwdArgs& a, const char* kt, const char* vt, const TileLane<DP>& ln,
                                         int key0, bool masked, const PageSlice* pages) {
    // one stage ahead at D = 128 with three row tiles (two spill), else two
    Ahead<DP == 128 && NQ == 3 ? 1 : 2> ko, vo;
    ko.preload([&](int i) { return row_operand<DP>(kt, ln, i / NC, i % NC); });
#pragma unroll
    for (int h = 0; h < H; ++h) {
      floatx4 x[2][NQ];
#pragma unroll
      for (int n = 0; n < NQ; ++n) x[0][n] = x[1][n] = floatx4{0, 0, 0, 0};
      stages<2 * NC>(
          ko, [&](int i) { return row_operand<DP>(kt, ln, 2 * h + i / NC, i % NC); },
          [&](int i, const uint4& k) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) x[i / NC][n] = mfma_qk<T>(k, q[n][i % NC], x[i / NC][n]);
          },
          vo, [&](int i) { return tr_operand<DP>(vt, ln, h, i); });
      uint4 w[NQ];
      weights(a, key0 + 32 * h, masked, pages, x, w);
      stages<NO>(
          vo, [&](int i) { return tr_operand<DP>(vt, ln, h, i); },
          [&](int i, const uint4& v) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) o[i][n] = mfma_qk<T>(v, w[n], o[i][n]);
          },
          ko, [&](int i) { return h + 1 < H ? row_operand<DP>(kt, ln, 2 * h + 2 + i / NC, i % NC) : uint4{}; });
    }
  }

  // Scores x of 32 keys to weights w, the offsets and sums brought up to date.
  __device__ __forceinline__ void weights(const AttnFwdArgs& a, int key0, bool masked, const PageSlice* pages,
                                          floatx4 (&x)[2][NQ], uint4 (&w)[NQ]) {
    const int g = (threadIdx.x & 63) >> 4;
    if (masked || (pages && pages->bad)) {
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int j = key0 + 16 * t + 4 * g + r;
          const bool nan = pages && pages->bad && pages->number(a.pg, min(j, max_key)) < 0;
#pragma unroll
          for (int n = 0; n < NQ; ++n) {
            x[t][n][r] = nan ? __builtin_nanf("") : x[t][n][r];
            x[t][n][r] = j >= lo[n] && j < hi[n] ? x[t][n][r] : -__builtin_inff();
          }
        }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      float mx = x[0][n][0];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, x[t][n][r]);
      if (__any(__builtin_fmaf(mx, a.c, -off[n]) > kOffsetLimit)) {
        mx *= a.c;
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const bool grow = mx - off[n] > kOffsetLimit;
        const float next = grow ? mx - kOffsetBelow : off[n];
        const float by = grow ? __builtin_amdgcn_exp2f(off[n] - next) : 1.0f;
        off[n] = next;
        sum[n] *= by;
#pragma unroll
        for (int ct = 0; ct < NO; ++ct) o[ct][n] *= by;
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          x[t][n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][n][r], a.c, -off[n]));
          sum[n] += x[t][n][r];
        }
      // weights rounded to the values' type (the matrix cores take nothing
      // wider): at most half a step, 2^-8 (bf16) or 2^-11 (fp16) of each; the sum of
      // weights is of the unrounded ones
      w[n] = uint4{pack2<T>(x[0][n][0], x[0][n][1]), pack2<T>(x[0][n][2], x[0][n][3]),
                   pack2<T>(x[1][n][0], x[1][n][1]), pack2<T>(x[1][n][2], x[1][n][3])};
    }
  }
  int max_key;  // the last key whose page number is at hand
};

// Results of columns c .. c + 3 of row r (o / sum of weights z, offset off; first:
// the thread that writes the row's own numbers): to the caller's arrays, or as
// part of a row whose keys are split.
template <typename T>
__device__ __forceinline__ void write_row(const AttnFwdArgs& a, const AttnJob& w, int r, int c, floatx4 o, float off,
                                          float z, bool first) {
  const AttnShape& s = a.s;
  if (r >= w.limit) return;
  const bool rest = r >= w.rows;
  if (rest && (!s.zero_rest || a.splits > 1)) return;  // (parts: k_attn_join sees to them)
  const int token = a.per > 1 ? r / a.per : r;
  const int h = a.per > 1 ? w.head * a.per + (r - token * a.per) : w.head;
  const int64_t row = w.sq.q0 + token;
  if (a.splits > 1) {
    const int64_t at = ((w.part * (int64_t)(s.packed ? 1 : s.B) + (s.packed ? 0 : w.b)) * s.M + row) * s.Hq + h;
    if (first) a.part_z[2 * at] = off, a.part_z[2 * at + 1] = z;
    if (off == kNoKeys) return;  // the sums are not looked at
    store_sums(a.part_o + at * s.C, c, s.C, o);
    return;
  }
  const bool empty = rest || off == kNoKeys;
  const float inv = 1.0f / z;
  floatx4 y;
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = empty ? 0.0f : between<T>(o[e] * inv);
  if (!rest || (s.zero_rest & kRestOut)) {
    store4<T>(a.out.p + w.b * a.out.sb + row * a.out.sr + h * a.out.sh, c, s.C, a.out.vec, y[0], y[1], y[2], y[3]);
    if (a.low.p)
      store4<T>(a.low.p + w.b * a.low.sb + row * a.low.sr + h * a.low.sh, c, s.C, a.low.vec, left<T>(y[0]),
                left<T>(y[1]), left<T>(y[2]), left<T>(y[3]));
  }
  if (first && a.lse && (!rest || (s.zero_rest & kRestLse)))
    a.lse[w.b * a.lse_sb + h * a.lse_sh + row] = empty ? -__builtin_inff() : (off + __builtin_amdgcn_logf(z)) * kLn2;
}

template <typename T, int DP, int NQ, int NW, bool PAGED, bool WIDE>
__global__ __launch_bounds__(64 * NW, 2) void k_attn_fwd(const AttnFwdArgs a) {
  constexpr int BK = attn_keys<DP>(), NO = DP / 16, TILE = BK * DP * 2, ROWS = 16 * NQ * NW;
  constexpr int NB = (NO * 4 + 31) / 32;
  __shared__ __align__(1024) char smem[2 * 2 * TILE];
  __shared__ int mark[4];
  // infinities that reach the lane's results: bit 4 ct + r of its column tile n
  __shared__ uint32_t inf_bits[64 * NW][2 * NQ * NB];
  __shared__ int32_t slice[PAGED ? kSlice : 1];
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);

  AttnJob job;
  if (!attn_job<ROWS, PAGED, true>(a, job)) return;
  const int kn = job.sq.kn, wr0 = job.r0 + wave * 16 * NQ;
  AttnRows<T, DP, NQ> rows;
  rows.start(a, job, wr0);
  const KeyRange all = keys_of_rows(a, job, job.r0, job.r0 + ROWS - 1);
  const KeyRange mine = keys_of_rows(a, job, wr0, wr0 + 16 * NQ - 1);
  int k_lo = all.lo, k_hi = all.hi;
  split_keys(a, job, BK, k_lo, k_hi);
  rows.start_offsets(k_lo, k_hi);

  const TileLane<DP> ln;
  const char* kb = a.k.p + (PAGED ? 0 : job.b * a.k.sb + (int64_t)job.sq.k0 * a.k.sr) + job.kvh * a.k.sh;
  const char* vb = a.v.p + (PAGED ? 0 : job.b * a.v.sb + (int64_t)job.sq.k0 * a.v.sr) + job.kvh * a.v.sh;
  const TileCopy<DP, BK, 64 * NW> tc(threadIdx.x);
  PageSlice pages;
  // Copies of a tile into a stage; rows past the last key repeat it (they are
  // masked, and stay in the array).
  auto issue = [&](int key0, int stage, int end) {
    char* t = smem + stage * 2 * TILE;
    auto key_of = [&](int i) { return min(key0 + tc.row0 + i * tc.STEP, kn - 1); };
    if constexpr (PAGED) {
      copy_pages<WIDE>(a, pages, tc, t, t + TILE, kb, vb, key0, end);
    } else if constexpr (WIDE) {
      tc.wide(t, kb + (int64_t)key0 * a.k.sr, (uint32_t)a.k.sr, kn - 1 - key0, s.D);
      tc.wide(t + TILE, vb + (int64_t)key0 * a.v.sr, (uint32_t)a.v.sr, kn - 1 - key0, s.C);
    } else {
      tc.narrow_rows(t, s.D, [&](int i) { return kb + (int64_t)key_of(i) * a.k.sr; });
      tc.narrow_rows(t + TILE, s.C, [&](int i) { return vb + (int64_t)key_of(i) * a.v.sr; });
    }
  };

  if (s.D < DP || s.C < DP) {
    clear_tiles<64 * NW>(smem, 2 * 2 * TILE);
    __syncthreads();
  }
  bool infinities = false;
  int it = 0;
  // keys in stretches whose page numbers fit in LDS (not paged: one stretch)
  const int64_t most = PAGED ? max((int64_t)(kSlice - 2) * a.pg.size / BK * BK, (int64_t)BK) : (int64_t)1 << 31;
  for (int from = k_lo; from < k_hi;) {
    const int to = (int)min(from + most, (int64_t)k_hi);
    if constexpr (PAGED) {
      if (from > k_lo) __syncthreads();  // nobody reads the last stretch's numbers
      pages.load(a.pg, slice, job.b, from, to, 64 * NW);
      rows.max_key = to - 1;
    }
    issue(from, 0, to);
    int stage = 0;
    for (int key0 = from; key0 < to; key0 += BK, stage ^= 1) {
      ++it;
      copies_done();
      const bool bordered = key0 + BK > all.in_hi || key0 < all.in_lo;
      if (bordered && clean_tile<T, DP, BK, 64 * NW>(smem + (stage * 2 + 1) * TILE, threadIdx.x)) mark[it & 3] = it;
      tile_barrier();  // this tile has landed everywhere, and nobody reads the other stage
      if (key0 + BK < to) issue(key0 + BK, stage ^ 1, to);
      if (bordered && uniform(mark[it & 3]) == it) {
        found_infinities<T, DP, BK, NQ, PAGED>(a, vb, job.b, kn, key0, rows.lo, rows.hi, inf_bits[threadIdx.x],
                                               !infinities);
        infinities = true;
      }
      if (key0 < mine.hi && key0 + BK > mine.lo) {
        const char* kt = smem + stage * 2 * TILE;
        const bool masked = key0 + BK > mine.in_hi || key0 < mine.in_lo;
        rows.template attend<BK / 32>(a, kt, kt + TILE, ln, key0, masked, PAGED ? &pages : nullptr);
      }
    }
    from = to;
  }

#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float z = rows.sum[n];
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
#pragma unroll
    for (int ct = 0; ct < NO; ++ct) {
      floatx4 y = rows.o[ct][n];
      if (infinities) add_infinities<NB>(inf_bits[threadIdx.x], n, ct, y);
      write_row<T>(a, job, wr0 + 16 * n + (lane & 15), 16 * ct + 4 * (lane >> 4), y, rows.off[n], z,
                   ct == 0 && lane < 16);
    }
  }
}

// The same for few rows (16 NQ, for instance the query heads that share a key head,
// of one new token): bound by reading the keys and values once, so the NW waves of a
// workgroup share the rows and take 32-key tiles in turn, each through a ring of its
// own (no barrier in the loop), and their sums are joined at the end.
template <typename T, int DP, int NQ, int NW, bool PAGED, bool WIDE>
__global__ __launch_bounds__(64 * NW) void k_attn_rows(const AttnFwdArgs a) {
  constexpr int NO = DP / 16, TILE = 32 * DP * 2, ROWS = 16 * NQ, NB = (NO * 4 + 31) / 32, NT = 64 * NW;
  constexpr int RING = NW * 2 * 2 * TILE, JOIN = NW * NQ * NO * 64 * 16;
  __shared__ __align__(1024) char smem[RING > JOIN ? RING : JOIN];
  __shared__ uint32_t inf_bits[NT][2 * NQ * NB];
  __shared__ int32_t slice[PAGED ? kSlice : 1];
  __shared__ float w_off[NW][ROWS], w_sum[NW][ROWS];
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);

  AttnJob job;
  if (!attn_job<ROWS, PAGED, false>(a, job)) return;
  const int kn = job.sq.kn;
  AttnRows<T, DP, NQ> rows;
  rows.start(a, job, job.r0);
  const KeyRange all = keys_of_rows(a, job, job.r0, job.r0 + ROWS - 1);
  int k_lo = all.lo, k_hi = all.hi;
  split_keys(a, job, 32, k_lo, k_hi);
  rows.start_offsets(k_lo, k_hi);

  const TileLane<DP> ln;
  const char* kb = a.k.p + (PAGED ? 0 : job.b * a.k.sb + (int64_t)job.sq.k0 * a.k.sr) + job.kvh * a.k.sh;
  const char* vb = a.v.p + (PAGED ? 0 : job.b * a.v.sb + (int64_t)job.sq.k0 * a.v.sr) + job.kvh * a.v.sh;
  const TileCopy<DP, 32, 64> tc(lane);
  char* ring = smem + wave * 4 * TILE;
  PageSlice pages;
  auto issue = [&](int key0, int stage, int end) {
    char* t = ring + stage * 2 * TILE;
    auto key_of = [&](int i) { return min(key0 + tc.row0 + i * tc.STEP, kn - 1); };
    if constexpr (PAGED) {
      copy_pages<WIDE>(a, pages, tc, t, t + TILE, kb, vb, key0, end);
    } else if constexpr (WIDE) {
      tc.wide(t, kb + (int64_t)key0 * a.k.sr, (uint32_t)a.k.sr, kn - 1 - key0, s.D);
      tc.wide(t + TILE, vb + (int64_t)key0 * a.v.sr, (uint32_t)a.v.sr, kn - 1 - key0, s.C);
    } else {
      tc.narrow_rows(t, s.D, [&](int i) { return kb + (int64_t)key_of(i) * a.k.sr; });
      tc.narrow_rows(t + TILE, s.C, [&](int i) { return vb + (int64_t)key_of(i) * a.v.sr; });
    }
  };

  if (s.D < DP || s.C < DP) {
    clear_tiles<NT>(smem, RING);
    __syncthreads();
  }
  bool infinities = false;
  const int64_t most = PAGED ? max((int64_t)(kSlice - 2) * a.pg.size / 32 * 32, (int64_t)32) : (int64_t)1 << 31;
  for (int from = k_lo; from < k_hi;) {
    const int to = (int)min(from + most, (int64_t)k_hi);
    if constexpr (PAGED) {
      if (from > k_lo) __syncthreads();
      pages.load(a.pg, slice, job.b, from, to, NT);
      rows.max_key = to - 1;
    }
    const int step = 32 * NW;
    if (from + 32 * wave < to) issue(from + 32 * wave, 0, to);
    int stage = 0;
    for (int key0 = from + 32 * wave; key0 < to; key0 += step, stage ^= 1) {
      copies_done();  // this tile has landed, and nothing reads the other stage
      if (key0 + step < to) issue(key0 + step, stage ^ 1, to);
      char* kt = ring + stage * 2 * TILE;
      const bool masked = key0 + 32 > all.in_hi || key0 < all.in_lo;
      if (masked && __any(clean_tile<T, DP, 32, 64>(kt + TILE, lane))) {
        found_infinities<T, DP, 32, NQ, PAGED>(a, vb, job.b, kn, key0, rows.lo, rows.hi, inf_bits[threadIdx.x],
                                               !infinities);
        infinities = true;
      }
      rows.template attend<1>(a, kt, kt + TILE, ln, key0, masked, PAGED ? &pages : nullptr);
    }
    from = to;
  }

  // join the waves' sums at the largest of their offsets
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float z = rows.sum[n];
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    if (lane < 16) w_off[wave][16 * n + lane] = rows.off[n], w_sum[wave][16 * n + lane] = z;
  }
  __syncthreads();  // also: every wave is done with its ring
  floatx4* join = reinterpret_cast<floatx4*>(smem);
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    float top = kNoKeys;
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, w_off[w][16 * n + (lane & 15)]);
    const float by = __builtin_amdgcn_exp2f(rows.off[n] - top);
#pragma unroll
    for (int ct = 0; ct < NO; ++ct) {
      floatx4 y = rows.o[ct][n] * by;
      if (infinities) add_infinities<NB>(inf_bits[threadIdx.x], n, ct, y);
      join[((wave * NQ + n) * NO + ct) * 64 + lane] = y;
    }
  }
  __syncthreads();
  for (int i = threadIdx.x; i < NQ * NO * 64; i += NT) {
    const int l = i & 63, n = i / (NO * 64), ct = (i >> 6) % NO, r = 16 * n + (l & 15);
    float top = kNoKeys, z = 0.0f;
    floatx4 y{0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < NW; ++w) top = fmaxf(top, w_off[w][r]);
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      z += w_sum[w][r] * __builtin_amdgcn_exp2f(w_off[w][r] - top);
      y += join[w * NQ * NO * 64 + i];
    }
    write_row<T>(a, job, job.r0 + r, 16 * ct + 4 * (l >> 4), y, top, z, ct == 0 && l < 16);
  }
}

// Joins the parts of rows whose keys were split: one wave a row and query head.
// Lane p holds part p's offset and sum (at most 64 parts); the columns go four a
// lane, and lanes left over take every second (fourth) part.
constexpr int kMostParts = 64;
template <typename T>
__global__ __launch_bounds__(256) void k_attn_join(const AttnFwdArgs a) {
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 63;
  const int64_t units = (int64_t)(s.packed ? 1 : s.B) * s.M * s.Hq;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= units) return;
  const int h = (int)(unit % s.Hq);
  const int64_t at = unit / s.Hq;
  const int b = s.packed ? 0 : (int)(at / s.M);
  const int64_t row = at - (int64_t)b * s.M;
  char* out = a.out.p + b * a.out.sb + row * a.out.sr + h * a.out.sh;
  char* low = a.low.p ? a.low.p + b * a.low.sb + row * a.low.sr + h * a.low.sh : nullptr;
  float* lse = a.lse ? a.lse + b * a.lse_sb + h * a.lse_sh + row : nullptr;
  if (s.packed) {
    if (!in_sequences(s.q_index, s.B, (int)row)) return;  // written, or left, by the main kernel
  } else if (s.q_index && row >= clampi(s.q_index[b], 0, s.M)) {
    if (s.zero_rest & kRestOut)
      for (int c = lane; c < s.C; c += 64) {
        reinterpret_cast<uint16_t*>(out)[c] = 0;
        if (low) reinterpret_cast<uint16_t*>(low)[c] = 0;
      }
    if (lse && lane == 0 && (s.zero_rest & kRestLse)) *lse = -__builtin_inff();
    return;
  }
  float off = kNoKeys, z = 0.0f;
  if (lane < a.splits) {
    const floatx2 p = *reinterpret_cast<const floatx2*>(a.part_z + 2 * (lane * units + unit));
    off = p[0], z = p[1];
  }
  float top = off;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
  const float w = __builtin_amdgcn_exp2f(off - top);
  z *= w;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) z += __shfl_xor(z, d);
  const bool empty = top == kNoKeys;
  const float inv = 1.0f / z;
  const int span = s.C > 128 ? 64 : s.C > 64 ? 32 : 16, groups = 64 / span, group = lane / span;
  const int c = 4 * (lane & (span - 1));
  floatx4 y{0, 0, 0, 0};
#pragma unroll 8
  for (int p0 = 0; p0 < a.splits; p0 += groups) {
    const int p = p0 + group;
    const float wp = __shfl(w, p & 63), op = __shfl(off, p & 63);
    // parts without keys hold no sums; one whose weight vanishes beside the others'
    // still counts: its sums may hold an infinity or NaN, and 0 times those is NaN
    if (p >= a.splits || c >= s.C || op == kNoKeys) continue;
    y += load_sums(a.part_o + (p * units + unit) * s.C, c, s.C) * wp;
  }
  for (int d = span; d < 64; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] += __shfl_xor(y[e], d);
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = empty ? 0.0f : between<T>(y[e] * inv);
  if (group == 0) {
    store4<T>(out, c, s.C, a.out.vec, y[0], y[1], y[2], y[3]);
    if (low) store4<T>(low, c, s.C, a.low.vec, left<T>(y[0]), left<T>(y[1]), left<T>(y[2]), left<T>(y[3]));
  }
  if (lse && lane == 0) *lse = empty ? -__builtin_inff() : (top + __builtin_amdgcn_logf(z)) * kLn2;
}

}  // namespace gs
