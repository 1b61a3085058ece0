// gs_attn_bwd.h -- softmax attention, backward.  With P = exp(scale S - lse)
// formed again from the scores, dP = dO V^T and delta_m = <dout_m, out_m>
// (out with what its rounding left, where the caller has it):
//   dV = P^T dO ,  dS = P (dP - delta) ,  dQ = scale dS K ,  dK = scale dS^T Q .
//
// Two passes over the pairs, so that every gradient is a sum in a fixed order in
// the registers of one wave (no atomics): k_attn_bwd<.., false> owns query columns
// and streams K and V (dQ), <.., true> owns key columns and streams Q and dO of all
// the query heads that share the key head (dK, dV).  Both form S and dP from the
// streamed rows on the MFMA rows and the wave's columns, and contract P and dS,
// rounded to the inputs' type, with the transposed streamed tiles.  Bound by the
// matrix cores at D = 128: 2 x 4096 tokens, 32 query and 8 key heads, no mask: dQ
// 737 us (1.12 PFLOP/s of its three products), dK and dV 970 us (1.13 of their four);
// by LDS reads at D = 256, where a wave owns one tile of 16 columns; at D = 64 the
// exponentials and conversions take half as long as the products (0.77).
#pragma once

#include "gs_attn_fwd.h"

namespace gs {

struct AttnBwdArgs {
  AttnShape s;
  AttnArray q, k, v, dout, dq, dk, dv;
  const float* lse2;       // lse log2 e
  const float* delta;
  int64_t st_sb, st_sh;    // elements: lse2 and delta of (sequence, head)
  int32_t tiles, heads;    // as in AttnFwdArgs
  float c;                 // scale log2 e
  int32_t splits;          // dK, dV: workgroups that share the query heads of a key head
  int32_t wgs;             // workgroups of one split
  int32_t part_width;      // twice the wider of D and C, rounded up to fours
  float* part;             // with several: splits x rows x key heads x part_width sums, of dK and then dV
};

// fp16: kernel weights enter dV times 2^15 (a weight of 2^-16, one key of 65536,
// would be subnormal), and dS times a power of two of every column's own, moved as
// the forward pass moves its offsets: where the column's largest |dS| so far times
// it exceeds 2^15, it is brought back to 2^13 or above and the sums are scaled with
// it.  Both are exact and taken out of the sums.  So dS is held to 2^-38 of the
// column's largest, whatever other columns, heads and sequences hold: an infinity or
// NaN spoils its own columns only.  bf16 has the exponents of fp32.
constexpr int kWeightShift = 15;
constexpr float kDsLimit = 0x1p15f;
constexpr int kDsExponent = 14;       // brought to [2^13, 2^14)
constexpr float kDsFirst = 0x1p100f;
template <typename T>
constexpr bool scaled() { return __is_same(T, F16); }

// e with x in [2^(e-1), 2^e).
__device__ __forceinline__ int exponent_of(float x) { return __builtin_amdgcn_frexp_expf(x); }

// lse in log2 units and delta.  16 lanes a row and head; bound by reading dout and out.
struct AttnPrepArgs {
  AttnShape s;
  AttnArray out, low, dout;  // low.p may be NULL
  const float* lse;
  float* lse2;
  float* delta;
  int64_t st_sb, st_sh;
  int64_t units;        // rows x query heads, all sequences
};

__device__ __forceinline__ bool row_used(const int32_t* index, int packed, int b, int i, int rows, int B) {
  if (!index) return true;
  return packed ? in_sequences(index, B, i) : i < clampi(index[b], 0, rows);
}

// Columns 8 lane .. of a row (16 lanes a row) as fp32, zero past the width.
template <typename T>
__device__ __forceinline__ void row8(const char* row, int vec, int width, int c, float (&x)[8]) {
  uint32_t y[8];
  if (vec) {
    uint4 z{0, 0, 0, 0};
    if (c < width) z = *reinterpret_cast<const uint4*>(row + 2 * c);
    const uint32_t w[4] = {z.x, z.y, z.z, z.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = (w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = c + e < width ? reinterpret_cast<const uint16_t*>(row)[c + e] : 0u;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = T::to_float((uint16_t)y[e]);
}

template <typename T>
__global__ __launch_bounds__(256) void k_attn_prep(const AttnPrepArgs a) {
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 15;
  for (int64_t unit = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); unit < a.units; unit += (int64_t)gridDim.x * 16) {
    const int h = (int)(unit % s.Hq);
    const int64_t row = unit / s.Hq;
    const int b = s.packed ? 0 : (int)(row / s.M), i = s.packed ? (int)row : (int)(row % s.M);
    float dot = 0.0f;
    for (int c = 8 * lane; c < s.C; c += 128) {
      float x[8], o[8];
      row8<T>(a.dout.p + b * a.dout.sb + i * a.dout.sr + h * a.dout.sh, a.dout.vec, s.C, c, x);
      row8<T>(a.out.p + b * a.out.sb + i * a.out.sr + h * a.out.sh, a.out.vec, s.C, c, o);
      if (a.low.p) {
        float l[8];
        row8<T>(a.low.p + b * a.low.sb + i * a.low.sr + h * a.low.sh, a.low.vec, s.C, c, l);
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] += l[e];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) dot = __builtin_fmaf(x[e], o[e], dot);
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) dot += __shfl_xor(dot, d);
    if (lane == 0) {
      const int64_t at = b * a.st_sb + h * a.st_sh + i;
      a.delta[at] = dot;
      a.lse2[at] = a.lse[at] * kLog2e;
    }
  }
}

template <typename T>
__device__ __forceinline__ bool row_not_finite(const char* row, int width) {
  constexpr uint32_t e = exponent_bits<T>();
  bool bad = false;
  for (int c = 0; c < width; ++c) bad |= (reinterpret_cast<const uint16_t*>(row)[c] & e) == e;
  return bad;
}

// Whether the column operands of dP lie in LDS instead of registers.
constexpr bool attn_bwd_lds(int DP, int NT, bool KV) { return KV && DP == 128 && NT == 2; }

template <typename T, int DP, int NT, int NW, bool KV, bool WIDE>
__global__ __launch_bounds__(64 * NW, 2) void k_attn_bwd(const AttnBwdArgs a) {
  constexpr bool WLDS = attn_bwd_lds(DP, NT, KV);
  constexpr int BR = WLDS ? 32 : attn_keys<DP>(), NC = DP / 32, NO = DP / 16, TILE = BR * DP * 2, COLS = 16 * NT * NW;
  __shared__ __align__(1024) char smem[4 * TILE];
  __shared__ __align__(16) float stat[2][2][BR];  // [stage][lse, delta][row]
  __shared__ int mark[4];
  __shared__ __align__(1024) char wcols[WLDS ? COLS * DP * 2 : 16];
  const AttnShape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;

  int tile, head, b;
  const int id = folded(blockIdx.x, gridDim.x), split = KV ? id / a.wgs : 0;
  block_place(id - split * a.wgs, a.heads, tile, head);
  const int rows_all = KV ? s.N : s.M;
  if (s.packed) {
    const int slot = tile;
    int n;
    b = packed_tile(KV ? s.k_index : s.q_index, s.B, rows_all, 1, COLS, slot, nullptr, tile, n);
    if (b == kNoRow) {
      if ((s.zero_rest & kRestOut) && split == 0) {
        const int part = slot - tile, parts = a.tiles - tile;
        const RestRows rest(KV ? s.k_index : s.q_index, s.B, rows_all);
        if (KV) {
          if (a.dk.p) zero_rest_rows(a.dk, head, s.D, rest, part, parts);
          if (a.dv.p) zero_rest_rows(a.dv, head, s.C, rest, part, parts);
        } else {
          zero_rest_rows(a.dq, head, s.D, rest, part, parts);
        }
      }
      return;
    }
    if (!KV) tile = n - 1 - tile;  // causal: late queries and early keys have most pairs
  } else {
    const int per_seq = a.heads / s.B;
    b = head / per_seq;
    head -= b * per_seq;
    if (!KV) tile = a.tiles - 1 - tile;  // causal: late queries and early keys have most pairs
  }
  const AttnSeq sq = seq_of(s, b);
  const int ahead = sq.kn - sq.qn;
  const int cn = KV ? sq.kn : sq.qn, c0 = KV ? sq.k0 : sq.q0;  // column points
  const int rn = KV ? sq.qn : sq.kn, x0 = KV ? sq.q0 : sq.k0;  // streamed rows
  const int limit = s.packed ? cn : rows_all;
  const int t0 = tile * COLS;
  if (t0 >= limit) return;
  const AttnArray &X = KV ? a.q : a.k, &Y = KV ? a.dout : a.v;
  const AttnArray &U = KV ? a.k : a.q, &W = KV ? a.v : a.dout;

  const int wc0 = t0 + wave * 16 * NT;
  int lo[NT], hi[NT];
  uint4 uo[NT][NC], wo[WLDS ? 1 : NT][NC];
  char* wmine = wcols + (WLDS ? wave * 16 * NT * DP * 2 : 0);
  float clse[NT], cdelta[NT];
  auto range = [&](int at, int& l, int& h) {
    if (KV)
      key_range(s, at, ahead, sq.qn, l, h);
    else
      query_range(s, at, ahead, sq.kn, l, h);
  };
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    lo[n] = hi[n] = 0;
    clse[n] = cdelta[n] = 0.0f;
    if (cn > 0) {
      const int at = min(wc0 + 16 * n + col, cn - 1);
      range(at, lo[n], hi[n]);
      const char* u = U.p + b * U.sb + (int64_t)(c0 + at) * U.sr + head * U.sh;
      const char* w = W.p + b * W.sb + (int64_t)(c0 + at) * W.sr + head * W.sh;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        uo[n][c] = column_operand<T>(u, U.vec, s.D, c, 0);
        const uint4 x = column_operand<T>(w, W.vec, s.C, c, 0);
        if (WLDS)
          *reinterpret_cast<uint4*>(wmine + (16 * n + col) * DP * 2 + ((4 * c + g) ^ swz(col)) * 16) = x;
        else
          wo[WLDS ? 0 : n][c] = x;
      }
      if (!KV) {
        const int64_t i = b * a.st_sb + head * a.st_sh + c0 + at;
        clse[n] = a.lse2[i];
        cdelta[n] = a.delta[i];
      }
    }
  }
  int r_lo = 0, r_hi = 0, w_lo = 0, w_hi = 0, in_lo = 0, in_hi = 0;
  int all_lo = 0, all_hi = 0;  // rows that every column of the workgroup sees
  if (cn > 0 && t0 < cn) {
    range(t0, r_lo, all_hi);
    range(min(t0 + COLS, cn) - 1, all_lo, r_hi);
    range(min(wc0, cn - 1), w_lo, in_hi);
    range(min(wc0 + 16 * NT, cn) - 1, in_lo, w_hi);
    if (wc0 >= cn) w_hi = w_lo = 0;
  }
  r_lo = r_lo / BR * BR;

  floatx4 du[NO][NT], dw[KV ? NO : 1][NT];
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int ct = 0; ct < NO; ++ct) {
      du[ct][n] = floatx4{0, 0, 0, 0};
      if (KV) dw[ct][n] = floatx4{0, 0, 0, 0};
    }
  float up[NT];  // fp16: what dS is multiplied by
#pragma unroll
  for (int n = 0; n < NT; ++n) up[n] = scaled<T>() ? kDsFirst : 1.0f;

  const TileLane<DP> ln;
  // the stream: tiles of rows [r_lo, r_hi), once for every query head (KV)
  const int heads = KV ? s.G / a.splits : 1, h0 = KV ? head * s.G + split * heads : head / s.G;
  const int steps = r_hi > r_lo ? (r_hi - r_lo + BR - 1) / BR : 0;
  const TileCopy<DP, BR, 64 * NW> tc(tid);
  auto issue = [&](int h, int row0, int stage) {
    char* t = smem + stage * 2 * TILE;
    const char* xb = X.p + b * X.sb + (int64_t)x0 * X.sr + (h0 + h) * X.sh;
    const char* yb = Y.p + b * Y.sb + (int64_t)x0 * Y.sr + (h0 + h) * Y.sh;
    if constexpr (WIDE) {
      tc.wide(t, xb + (int64_t)row0 * X.sr, (uint32_t)X.sr, rn - 1 - row0, s.D);
      tc.wide(t + TILE, yb + (int64_t)row0 * Y.sr, (uint32_t)Y.sr, rn - 1 - row0, s.C);
    } else {
      auto row_of = [&](int i) { return min(row0 + tc.row0 + i * tc.STEP, rn - 1); };
      tc.narrow_rows(t, s.D, [&](int i) { return xb + (int64_t)row_of(i) * X.sr; });
      tc.narrow_rows(t + TILE, s.C, [&](int i) { return yb + (int64_t)row_of(i) * Y.sr; });
    }
    if (KV && wave < 2 && lane < BR) {  // the first wave copies lse, the second delta
      const float* p = (wave ? a.delta : a.lse2) + b * a.st_sb + (h0 + h) * a.st_sh + x0 + row0;
      copy4(p, min(lane, rn - 1 - row0) * 4, uniform(lds_offset(stat[stage][wave])));
    }
  };
  if (s.D < DP || s.C < DP) {
    clear_tiles<64 * NW>(smem, 4 * TILE);
    __syncthreads();
  }
  // columns that see a row with an infinity or NaN: their gradients are NaN
  bool spoilt[NT] = {};
  if (steps > 0) issue(0, r_lo, 0);
  int stage = 0, it = 0;
  for (int h = 0; h < heads; ++h)
    for (int st = 0; st < steps; ++st, stage ^= 1) {
      ++it;
      copies_done();
      const int row0 = r_lo + st * BR;
      const bool bordered = row0 + BR > all_hi || row0 < all_lo;
      if (bordered) {
        char* t = smem + stage * 2 * TILE;
        const bool x_bad = clean_tile<T, DP, BR, 64 * NW>(t, tid);
        const bool y_bad = clean_tile<T, DP, BR, 64 * NW>(t + TILE, tid);
        if (x_bad || y_bad) mark[it & 3] = it;
      }
      tile_barrier();
      if (st + 1 < steps)
        issue(h, r_lo + (st + 1) * BR, stage ^ 1);
      else if (h + 1 < heads)
        issue(h + 1, r_lo, stage ^ 1);
      if (bordered && uniform(mark[it & 3]) == it) {
        const int at = min(row0 + lane, rn - 1);
        const char* xr = X.p + b * X.sb + (int64_t)(x0 + at) * X.sr + (h0 + h) * X.sh;
        const char* yr = Y.p + b * Y.sb + (int64_t)(x0 + at) * Y.sr + (h0 + h) * Y.sh;
        const bool own = lane < BR && row0 + lane < rn;
        const uint64_t bad = __ballot(own && (row_not_finite<T>(xr, s.D) || row_not_finite<T>(yr, s.C)));
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const int f = clampi(lo[n] - row0, 0, BR), l = clampi(hi[n] - row0, f, BR);
          const uint64_t seen = (l == 64 ? ~0ull : (1ull << l) - 1) & ~(f == 64 ? ~0ull : (1ull << f) - 1);
          spoilt[n] |= (bad & seen) != 0;
        }
      }
      if (row0 >= w_hi || row0 + BR <= w_lo) continue;
      const char* xt = smem + stage * 2 * TILE;
      const char* yt = xt + TILE;
      const bool masked = row0 + BR > in_hi || row0 < in_lo;
#pragma unroll
      for (int hf = 0; hf < BR / 32; ++hf) {
        uint32_t pw[NT][4], dsw[NT][4];
        floatx4 sc2[2][NT], dp2[2][NT];
        // dP - delta: the sums start at -delta
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            sc2[t][n] = floatx4{0, 0, 0, 0};
            dp2[t][n] = KV ? -*reinterpret_cast<const floatx4*>(&stat[stage][1][32 * hf + 16 * t + 4 * g])
                           : floatx4{-cdelta[n], -cdelta[n], -cdelta[n], -cdelta[n]};
          }
        Ahead<2> xo, yo;
        auto load_x = [&](int t, int c) { return row_operand<DP>(xt, ln, 2 * hf + t, c); };
        auto load_y = [&](int t, int c) { return row_operand<DP>(yt, ln, 2 * hf + t, c); };
        auto load_ytr = [&](int i) { return tr_operand<DP>(yt, ln, hf, i); };
        auto load_xtr = [&](int i) { return tr_operand<DP>(xt, ln, hf, i); };
        xo.preload([&](int i) { return load_x(0, i); });
        if constexpr (WLDS) {
          // S of both row tiles, then dP with the operands of V from LDS
          stages<2 * NC>(
              xo, [&](int i) { return load_x(i / NC, i % NC); },
              [&](int i, const uint4& x) {
#pragma unroll
                for (int n = 0; n < NT; ++n) sc2[i / NC][n] = mfma_qk<T>(x, uo[n][i % NC], sc2[i / NC][n]);
              },
              yo, NoLoad{});
          uint4 y[2][2], w[2][NT];
          auto read = [&](int c) {
#pragma unroll
            for (int n = 0; n < NT; ++n) w[c & 1][n] = row_operand<DP>(wmine, ln, n, c);
#pragma unroll
            for (int t = 0; t < 2; ++t) y[c & 1][t] = load_y(t, c);
          };
          read(0);
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (c + 1 < NC) read(c + 1);
            stage_fence();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int n = 0; n < NT; ++n) dp2[t][n] = mfma_qk<T>(y[c & 1][t], w[c & 1][n], dp2[t][n]);
            stage_fence();
          }
          yo.preload(load_ytr);
          stage_fence();
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          floatx4(&sc)[NT] = sc2[t], (&dp)[NT] = dp2[t];
          floatx4 rl{0, 0, 0, 0};
          if (KV) rl = *reinterpret_cast<const floatx4*>(&stat[stage][0][32 * hf + 16 * t + 4 * g]);
          if constexpr (!WLDS) {
            stages<NC>(
                xo, [&](int i) { return load_x(t, i); },
                [&](int i, const uint4& x) {
#pragma unroll
                  for (int n = 0; n < NT; ++n) sc[n] = mfma_qk<T>(x, uo[n][i], sc[n]);
                },
                yo, [&](int i) { return load_y(t, i); });
            // what is read ahead of the exponentials: the next row tile's rows, or the
            // first transposed operands (of dO for dV, of K for dQ)
            stages<NC>(
                yo, [&](int i) { return load_y(t, i); },
                [&](int i, const uint4& y) {
#pragma unroll
                  for (int n = 0; n < NT; ++n) dp[n] = mfma_qk<T>(y, wo[WLDS ? 0 : n][i], dp[n]);
                },
                xo, [&](int i) { return t == 0 ? load_x(1, i) : KV ? load_ytr(i) : load_xtr(i); });
          }
#pragma unroll
          for (int n = 0; n < NT; ++n) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][r], a.c, -(KV ? rl[r] : clse[n])));
              float d = p * dp[n][r];
              if (masked) {
                const int j = row0 + 32 * hf + 16 * t + 4 * g + r;
                const bool in = j >= lo[n] && j < hi[n];
                p = in ? p : 0.0f;
                d = in ? d : 0.0f;
              }
              // the weights and dS are rounded to the inputs' type for the matrix cores
              sc[n][r] = scaled<T>() ? p * (float)(1 << kWeightShift) : p;
              dp[n][r] = d;
            }
            pw[n][2 * t] = pack2<T>(sc[n][0], sc[n][1]);
            pw[n][2 * t + 1] = pack2<T>(sc[n][2], sc[n][3]);
            if (!scaled<T>()) {
              dsw[n][2 * t] = pack2<T>(dp[n][0], dp[n][1]);
              dsw[n][2 * t + 1] = pack2<T>(dp[n][2], dp[n][3]);
            }
          }
        }
        if constexpr (scaled<T>()) {
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float mx = 0.0f;
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int r = 0; r < 4; ++r) mx = fmaxf(mx, __builtin_fabsf(dp2[t][n][r]));
            if (__any(mx * up[n] > kDsLimit)) {
              mx = fmaxf(mx, __shfl_xor(mx, 16));
              mx = fmaxf(mx, __shfl_xor(mx, 32));
              // (an infinity spoils its column anyway)
              const bool grow = mx * up[n] > kDsLimit && mx < __builtin_inff();
              const int e = grow ? kDsExponent - exponent_of(mx) : exponent_of(up[n]) - 1;
              const float by = __builtin_ldexpf(1.0f, e - (exponent_of(up[n]) - 1));
              up[n] = __builtin_ldexpf(1.0f, e);
#pragma unroll
              for (int ct = 0; ct < NO; ++ct) du[ct][n] *= by;
            }
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
              for (int r = 0; r < 2; ++r)
                dsw[n][2 * t + r] = pack2<T>(dp2[t][n][2 * r] * up[n], dp2[t][n][2 * r + 1] * up[n]);
          }
        }
        uint4 pb[NT], db[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          pb[n] = uint4{pw[n][0], pw[n][1], pw[n][2], pw[n][3]};
          db[n] = uint4{dsw[n][0], dsw[n][1], dsw[n][2], dsw[n][3]};
        }
        Ahead<2>& first = WLDS ? yo : xo;
        if constexpr (KV)
          stages<NO>(
              first, load_ytr,
              [&](int i, const uint4& y) {
#pragma unroll
                for (int n = 0; n < NT; ++n) dw[KV ? i : 0][n] = mfma_qk<T>(y, pb[n], dw[KV ? i : 0][n]);
              },
              WLDS ? xo : yo, load_xtr);
        stages<NO>(
            KV && !WLDS ? yo : xo, load_xtr,
            [&](int i, const uint4& x) {
#pragma unroll
              for (int n = 0; n < NT; ++n) du[i][n] = mfma_qk<T>(x, db[n], du[i][n]);
            },
            first, NoLoad{});
      }
    }

  const float w_scale = scaled<T>() ? 1.0f / (1 << kWeightShift) : 1.0f;
  const AttnArray& DU = KV ? a.dk : a.dq;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int at = wc0 + 16 * n + col;
    if (at >= limit || (at >= cn && (!(s.zero_rest & kRestOut) || split > 0))) continue;
    const bool none = at >= cn;
    const float down = scaled<T>() ? __builtin_ldexpf(1.0f, 1 - exponent_of(up[n])) : 1.0f;
    if (KV && a.splits > 1 && !none) {
      const int64_t row = (s.packed ? 0 : (int64_t)b * s.N) + c0 + at, rows = (int64_t)(s.packed ? 1 : s.B) * s.N;
      float* p = a.part + ((split * rows + row) * s.Hkv + head) * a.part_width;
#pragma unroll
      for (int ct = 0; ct < NO; ++ct) {
        const float nan = spoilt[n] ? __builtin_nanf("") : 0.0f;
        store_sums(p, 16 * ct + 4 * g, s.D, du[ct][n] * down * s.scale + nan);
        store_sums(p + a.part_width / 2, 16 * ct + 4 * g, s.C, dw[KV ? ct : 0][n] * w_scale + nan);
      }
      continue;
    }
    if (DU.p) {
      char* p = DU.p + b * DU.sb + (int64_t)(c0 + at) * DU.sr + head * DU.sh;
#pragma unroll
      for (int ct = 0; ct < NO; ++ct) {
        floatx4 y = du[ct][n] * down * s.scale;
        if (spoilt[n]) y = floatx4{1, 1, 1, 1} * __builtin_nanf("");
        if (none) y = floatx4{0, 0, 0, 0};
        store4<T>(p, 16 * ct + 4 * g, s.D, DU.vec, y[0], y[1], y[2], y[3]);
      }
    }
    if (KV && a.dv.p) {
      char* p = a.dv.p + b * a.dv.sb + (int64_t)(c0 + at) * a.dv.sr + head * a.dv.sh;
#pragma unroll
      for (int ct = 0; ct < NO; ++ct) {
        floatx4 y = dw[KV ? ct : 0][n] * w_scale;
        if (spoilt[n]) y = floatx4{1, 1, 1, 1} * __builtin_nanf("");
        if (none) y = floatx4{0, 0, 0, 0};
        store4<T>(p, 16 * ct + 4 * g, s.C, a.dv.vec, y[0], y[1], y[2], y[3]);
      }
    }
  }
}

// dk and dv from the sums of the workgroups that shared a key head: one wave a row
// and key head.
template <typename T>
__global__ __launch_bounds__(256) void k_attn_sum(const AttnBwdArgs a) {
  const AttnShape& s = a.s;
  const int64_t rows = (int64_t)(s.packed ? 1 : s.B) * s.N, units = rows * s.Hkv;
  const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (unit >= units) return;
  const int h = (int)(unit % s.Hkv), c = 4 * (threadIdx.x & 63);
  const int64_t at = unit / s.Hkv;
  const int b = s.packed ? 0 : (int)(at / s.N);
  const int64_t row = at - (int64_t)b * s.N;
  // rows of no sequence are written, or left, by the main kernel
  if (!row_used(s.k_index, s.packed, b, (int)row, s.N, s.B)) return;
  floatx4 x{0, 0, 0, 0}, y{0, 0, 0, 0};
  for (int p = 0; p < a.splits; ++p) {
    const float* from = a.part + (p * units + unit) * a.part_width;
    x += load_sums(from, c, s.D);
    y += load_sums(from + a.part_width / 2, c, s.C);
  }
  if (a.dk.p) store4<T>(a.dk.p + b * a.dk.sb + row * a.dk.sr + h * a.dk.sh, c, s.D, a.dk.vec, x[0], x[1], x[2], x[3]);
  if (a.dv.p) store4<T>(a.dv.p + b * a.dv.sb + row * a.dv.sr + h * a.dv.sh, c, s.C, a.dv.vec, y[0], y[1], y[2], y[3]);
}

}  // namespace gs
