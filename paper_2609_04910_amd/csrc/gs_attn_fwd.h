// gs_attn_fwd.h -- softmax attention, forward:
//   out_m = sum_n w_mn v_n / sum_n w_mn ,  w_mn = exp(scale q_m.k_n) ,
//   lse_m = log sum_n w_mn ,
// over the keys n that row m sees, in one pass: the weights are taken relative to
// a running offset o_m of the exponent (log2 units), and where a row's largest
// exponent outgrows it the sums so far are scaled by exp2(old - new).
//
// A workgroup of NW waves streams 64-key (DP = 256: 32-key) tiles of K and V
// through a two-stage LDS ring, one barrier a tile; wave w owns 16*NQ rows whose
// query operands and output sums stay in registers.
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
};

// Weights lie below 2^15 relative to the offset, the largest of a row between
// 2^7 and 2^15: fp16 then holds weights down to 2^-21 of the largest in full
// precision, and the sums are scaled again only where the largest exponent grows
// by more than 8.
constexpr float kOffsetBelow = 7.0f;
constexpr float kOffsetLimit = 15.0f;
constexpr float kNoOffset = -3.0e38f;

// Page number of key j of sequence b, and the address of the key's row in a page;
// NULL for a number outside the cache.
__device__ __forceinline__ int page_of(const AttnPages& pg, int b, int j) {
  const int pi = pg.shift >= 0 ? j >> pg.shift : (int)((uint32_t)j / (uint32_t)pg.size);
  return pg.table[(int64_t)b * pg.width + pi];
}
__device__ __forceinline__ const char* page_row(const AttnPages& pg, const char* base, int64_t page_stride, int64_t sr,
                                                int page, int j) {
  const int off = pg.shift >= 0 ? j & (pg.size - 1) : (int)((uint32_t)j % (uint32_t)pg.size);
  if ((uint32_t)page >= (uint32_t)pg.pages) return nullptr;
  return base + page * page_stride + off * sr;
}

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

// Sets the bits of the lane's results that infinities among the values of a tile
// reach: +inf in the first NB words of each column tile, -inf in the next, NaN in
// both (inf - inf is NaN).  The values are
// read from the caller's array again; products of indicators tell which columns
// see a row that has one.
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
        const char* p = PAGED ? page_row(a.pg, vb, a.pg.page_stride_v, a.v.sr, page_of(a.pg, b, j), j)
                              : vb + (int64_t)j * a.v.sr;
        const uint32_t x = p && c < a.s.C ? reinterpret_cast<const uint16_t*>(p)[c] : 0u;
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

template <typename T, int DP, int NQ, int NW, bool PAGED, bool WIDE>
__global__ __launch_bounds__(64 * NW, 2) void k_attn_fwd(const AttnFwdArgs a) {
  constexpr int BK = attn_keys<DP>(), NC = DP / 32, NO = DP / 16, TILE = BK * DP * 2, ROWS = 16 * NQ * NW;
  __shared__ __align__(1024) char smem[4 * TILE];
  __shared__ int mark[4];
  // infinities that reach the lane's results: bit 4 ct + r of its column tile n
  constexpr int NB = (NO * 4 + 31) / 32;
  __shared__ uint32_t inf_bits[64 * NW][2 * NQ * NB];
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int col = lane & 15, g = lane >> 4;

  int tile, head, b;
  block_place(blockIdx.x, a.heads, tile, head);
  if (s.packed) {
    const int slot = a.tiles - 1 - tile;
    b = packed_tile(s.q_index, s.B, s.M, a.per, ROWS, slot, tile);
    if (b == kNoRow) {  // slots past the last tile: rows of no sequence
      if (s.zero_rest) {
        const int part = slot - tile, parts = a.tiles - tile;
        const int end = s.B > 0 ? clampi(s.q_index[s.B], 0, s.M) : 0;
        for (int h = head * a.per; h < (head + 1) * a.per; ++h) {
          if (s.zero_rest & kRestOut) {
            zero_rows(a.out, 0, h, s.C, end, s.M, part, parts);
            if (a.low.p) zero_rows(a.low, 0, h, s.C, end, s.M, part, parts);
          }
          if (a.lse && (s.zero_rest & kRestLse))
            for (int64_t r = end + part; r < s.M; r += parts)
              if (threadIdx.x == 0) a.lse[h * a.lse_sh + r] = -__builtin_inff();
        }
      }
      return;
    }
  } else {
    const int per_seq = a.heads / s.B;
    b = head / per_seq;
    head -= b * per_seq;
    tile = a.tiles - 1 - tile;  // the tiles that see most keys first
  }
  const int kvh = a.per > 1 ? head : head / s.G;
  AttnSeq sq;
  if (PAGED) {
    if (s.packed)
      seq_side(s.q_index, 1, b, s.M, sq.q0, sq.qn);
    else
      sq.q0 = 0, sq.qn = s.M;
    sq.k0 = 0;
    sq.kn = clampi(a.pg.lens[b], 0, (int)min((int64_t)a.pg.width * a.pg.size, (int64_t)0x3fffffff));
    sq.q0 = uniform(sq.q0), sq.qn = uniform(sq.qn), sq.kn = uniform(sq.kn);
  } else {
    sq = seq_of(s, b);
  }
  const int ahead = sq.kn - sq.qn;
  const int rows = sq.qn * a.per;          // rows of this head group
  const int limit = s.packed ? rows : s.M * a.per;  // and rows that the call owns
  const int r0 = tile * ROWS;
  if (r0 >= limit) return;

  // the wave's rows: token and head of the lane's column in each of its tiles;
  // rows past the end repeat the last one (nothing of them is written)
  const int wr0 = r0 + wave * 16 * NQ;
  int lo[NQ], hi[NQ];
  uint4 qo[NQ][NC];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = min(wr0 + 16 * n + col, rows - 1);
    const int token = a.per > 1 ? r / a.per : r;
    const int h = a.per > 1 ? head * a.per + (r - token * a.per) : head;
    lo[n] = hi[n] = 0;
    if (rows > 0) {
      query_range(s, token, ahead, sq.kn, lo[n], hi[n]);
      const char* p = a.q.p + b * a.q.sb + (int64_t)(sq.q0 + token) * a.q.sr + h * a.q.sh;
#pragma unroll
      for (int c = 0; c < NC; ++c) qo[n][c] = column_operand<T>(p, a.q.vec, s.D, c, a.neg);
    }
  }
  // key ranges of the workgroup and of the wave (token ranges are monotone)
  int k_lo = 0, k_hi = 0, w_lo = 0, w_hi = 0, in_lo = 0, in_hi = 0;
  int all_lo = 0, all_hi = 0;  // keys that every row of the workgroup sees
  if (rows > 0 && r0 < rows) {
    query_range(s, r0 / a.per, ahead, sq.kn, k_lo, all_hi);
    query_range(s, (min(r0 + ROWS, rows) - 1) / a.per, ahead, sq.kn, all_lo, k_hi);
    const int f = min(wr0, rows - 1) / a.per, l = min(wr0 + 16 * NQ - 1, rows - 1) / a.per;
    query_range(s, f, ahead, sq.kn, w_lo, in_hi);
    query_range(s, l, ahead, sq.kn, in_lo, w_hi);
    if (wr0 >= rows) w_hi = w_lo = 0;
  }
  k_lo = k_lo / BK * BK;

  floatx4 o[NO][NQ];
  float off[NQ], sum[NQ];
#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    off[n] = kNoOffset;
    sum[n] = 0.0f;
#pragma unroll
    for (int ct = 0; ct < NO; ++ct) o[ct][n] = floatx4{0, 0, 0, 0};
  }

  const TileLane<DP> ln;
  const char* kb = a.k.p + (PAGED ? 0 : b * a.k.sb + (int64_t)sq.k0 * a.k.sr) + kvh * a.k.sh;
  const char* vb = a.v.p + (PAGED ? 0 : b * a.v.sb + (int64_t)sq.k0 * a.v.sr) + kvh * a.v.sh;
  // Copies of a tile into a stage; rows past the last key repeat it (they are
  // masked, and stay in the array).  Page numbers are read a tile ahead: waiting
  // for them between a tile's copies would wait for the copies too.
  const TileCopy<DP, BK, 64 * NW> tc;
  int pages[PAGED ? TileCopy<DP, BK, 64 * NW>::N : 1];
  auto key_of = [&](int key0, int i) { return min(key0 + tc.row0 + i * tc.STEP, sq.kn - 1); };
  auto read_pages = [&](int key0) {
    if constexpr (PAGED) {
#pragma unroll
      for (int i = 0; i < tc.N; ++i) pages[i] = page_of(a.pg, b, key_of(key0, i));
    }
  };
  auto issue = [&](int key0, int stage) {
    char* t = smem + stage * 2 * TILE;
    if constexpr (PAGED) {
      auto krow = [&](int i) { return page_row(a.pg, kb, a.pg.page_stride_k, a.k.sr, pages[i], key_of(key0, i)); };
      auto vrow = [&](int i) { return page_row(a.pg, vb, a.pg.page_stride_v, a.v.sr, pages[i], key_of(key0, i)); };
      if constexpr (WIDE) {
        tc.wide_rows(t, s.D, krow);
        tc.wide_rows(t + TILE, s.C, vrow);
      } else {
        tc.narrow_rows(t, s.D, krow);
        tc.narrow_rows(t + TILE, s.C, vrow);
      }
      if (key0 + BK < k_hi) read_pages(key0 + BK);
    } else if constexpr (WIDE) {
      tc.wide(t, kb + (int64_t)key0 * a.k.sr, (uint32_t)a.k.sr, sq.kn - 1 - key0, s.D);
      tc.wide(t + TILE, vb + (int64_t)key0 * a.v.sr, (uint32_t)a.v.sr, sq.kn - 1 - key0, s.C);
    } else {
      tc.narrow_rows(t, s.D, [&](int i) { return kb + (int64_t)key_of(key0, i) * a.k.sr; });
      tc.narrow_rows(t + TILE, s.C, [&](int i) { return vb + (int64_t)key_of(key0, i) * a.v.sr; });
    }
  };

  if (s.D < DP || s.C < DP) {
    clear_tiles<64 * NW>(smem, 4 * TILE);
    __syncthreads();
  }
  bool infinities = false;
  if (k_lo < k_hi) {
    read_pages(k_lo);
    issue(k_lo, 0);
  }
  int stage = 0;
  for (int key0 = k_lo, it = 1; key0 < k_hi; key0 += BK, stage ^= 1, ++it) {
    const bool bordered = key0 + BK > all_hi || key0 < all_lo;
    if (bordered) {
      copies_done();
      if (clean_tile<T, DP, BK, 64 * NW>(smem + (stage * 2 + 1) * TILE)) mark[it & 3] = it;
    }
    tile_barrier();  // this tile has landed, and nobody reads the other stage
    if (key0 + BK < k_hi) issue(key0 + BK, stage ^ 1);
    if (bordered && uniform(mark[it & 3]) == it) {
      found_infinities<T, DP, BK, NQ, PAGED>(a, vb, b, sq.kn, key0, lo, hi, inf_bits[threadIdx.x], !infinities);
      infinities = true;
    }
    if (key0 >= w_hi || key0 + BK <= w_lo) continue;
    const char* kt = smem + stage * 2 * TILE;
    const char* vt = kt + TILE;
    const bool masked = key0 + BK > in_hi || key0 < in_lo;
#pragma unroll
    for (int h = 0; h < BK / 32; ++h) {
      floatx4 x[2][NQ];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
#pragma unroll
        for (int n = 0; n < NQ; ++n) x[t][n] = floatx4{0, 0, 0, 0};
        scores<T, DP, NQ>(kt, ln, 2 * h + t, qo, x[t]);
      }
      if (masked) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const int j = key0 + 32 * h + 16 * t + 4 * g + r;
              x[t][n][r] = j >= lo[n] && j < hi[n] ? x[t][n][r] : -__builtin_inff();
            }
      }
      uint4 w[NQ];
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
        // wider): at most 2^-9 (bf16) or 2^-12 (fp16) of each; the sum of weights
        // is of the unrounded ones
        w[n] = uint4{pack2<T>(x[0][n][0], x[0][n][1]), pack2<T>(x[0][n][2], x[0][n][3]),
                     pack2<T>(x[1][n][0], x[1][n][1]), pack2<T>(x[1][n][2], x[1][n][3])};
      }
      contract<T, DP>(vt, ln, h, w, o);
    }
  }

#pragma unroll
  for (int n = 0; n < NQ; ++n) {
    const int r = wr0 + 16 * n + col;
    float z = sum[n];
    z += __shfl_xor(z, 16);
    z += __shfl_xor(z, 32);
    if (r >= limit || (r >= rows && !s.zero_rest)) continue;
    const int tk = a.per > 1 ? r / a.per : r;
    const int h = a.per > 1 ? head * a.per + (r - tk * a.per) : head;
    if (r >= rows) z = 0.0f;
    const bool empty = z == 0.0f;
    const float inv = empty ? 0.0f : 1.0f / z;
    char* p = a.out.p + b * a.out.sb + (int64_t)(sq.q0 + tk) * a.out.sr + h * a.out.sh;
    char* pl = a.low.p ? a.low.p + b * a.low.sb + (int64_t)(sq.q0 + tk) * a.low.sr + h * a.low.sh : nullptr;
    const bool rest = r >= rows;
#pragma unroll
    for (int ct = 0; ct < NO; ++ct) {
      if (rest && !(s.zero_rest & kRestOut)) break;
      floatx4 y = o[ct][n];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t bit = 1u << ((4 * ct + e) & 31);
        y[e] = empty ? 0.0f : y[e] * inv;
        if (infinities) {
          if (inf_bits[threadIdx.x][2 * n * NB + ct / 8] & bit) y[e] += __builtin_inff();
          if (inf_bits[threadIdx.x][(2 * n + 1) * NB + ct / 8] & bit) y[e] -= __builtin_inff();
        }
      }
      store4<T>(p, 16 * ct + 4 * g, s.C, a.out.vec, y[0], y[1], y[2], y[3]);
      if (pl)
        store4<T>(pl, 16 * ct + 4 * g, s.C, a.low.vec, left<T>(y[0]), left<T>(y[1]), left<T>(y[2]), left<T>(y[3]));
    }
    if (a.lse && g == 0 && (!rest || (s.zero_rest & kRestLse)))
      a.lse[b * a.lse_sb + h * a.lse_sh + sq.q0 + tk] =
          empty ? -__builtin_inff() : (off[n] + __builtin_amdgcn_logf(z)) * kLn2;
  }
}

}  // namespace gs
