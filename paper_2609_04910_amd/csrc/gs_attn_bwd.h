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
// rounded to the inputs' type, with the transposed streamed tiles.
#pragma once

#include "gs_attn_fwd.h"

namespace gs {

struct AttnBwdArgs {
  AttnShape s;
  AttnArray q, k, v, dout, dq, dk, dv;
  const float* lse;
  const float* delta;
  int64_t st_sb, st_sh;    // elements: lse and delta of (sequence, head)
  const uint32_t* norms;   // fp16: bits of the largest row norms of dout and v
  int32_t tiles, heads;    // as in AttnFwdArgs
  float c;                 // scale log2 e
};

// fp16: kernel weights enter dV times 2^15 (a weight of 2^-16, one key of 65536,
// would be subnormal), and dS times 2^e with the largest possible |dS|, twice the
// product of the row norms of dout and v, below 2^15; both exact, taken out of the
// sums.  bf16 has the exponents of fp32.
constexpr int kWeightShift = 15;
template <typename T>
constexpr bool scaled() { return __is_same(T, F16); }

__device__ __forceinline__ int ds_exponent(const uint32_t* norms) {
  const float x = __builtin_bit_cast(float, norms[0]), y = __builtin_bit_cast(float, norms[1]);
  const float z = x * y;
  if (!(z > 0.0f) || !(z < __builtin_inff())) return 0;
  int e;
  (void)frexpf(z, &e);  // z < 2^e
  return clampi(14 - e, -100, 100);
}

// delta, and for fp16 the largest row norms of dout (norms[0]) and v (norms[1])
// over the rows in use.  16 lanes a row and head; a maximum of non-negative
// numbers by their bits does not depend on its order.
template <typename T>
__device__ __forceinline__ float elem(const char* row, int c) {
  return T::to_float(reinterpret_cast<const uint16_t*>(row)[c]);
}

struct AttnPrepArgs {
  AttnShape s;
  AttnArray out, low, dout, v;  // low.p may be NULL
  float* delta;
  int64_t st_sb, st_sh;
  uint32_t* norms;      // NULL: not wanted
  int64_t q_units;      // rows x query heads, all sequences (padded to whole workgroups by the grid)
  int64_t k_units;      // rows x key heads (0: no norms)
  int32_t q_blocks;
};

__device__ __forceinline__ bool row_used(const int32_t* index, int packed, int b, int i, int rows, int B) {
  if (!index) return true;
  if (!packed) return i < clampi(index[b], 0, rows);
  return B > 0 && i >= index[0] && i < index[B];
}

template <typename T>
__global__ __launch_bounds__(256) void k_attn_prep(const AttnPrepArgs a) {
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 15;
  const bool keys = (int)blockIdx.x >= a.q_blocks;
  const int64_t unit = (int64_t)(blockIdx.x - (keys ? a.q_blocks : 0)) * 16 + (threadIdx.x >> 4);
  float norm = 0.0f;
  if (unit < (keys ? a.k_units : a.q_units)) {
    const int H = keys ? s.Hkv : s.Hq, R = keys ? s.N : s.M;
    const int h = (int)(unit % H);
    const int64_t row = unit / H;
    const int b = s.packed ? 0 : (int)(row / R), i = s.packed ? (int)row : (int)(row % R);
    const bool used = row_used(keys ? s.k_index : s.q_index, s.packed, b, i, R, s.B);
    float dot = 0.0f, sq = 0.0f;
    if (keys) {
      const char* p = a.v.p + b * a.v.sb + i * a.v.sr + h * a.v.sh;
      for (int c = lane; c < s.C; c += 16) {
        const float x = elem<T>(p, c);
        sq = __builtin_fmaf(x, x, sq);
      }
    } else {
      const char* p = a.dout.p + b * a.dout.sb + i * a.dout.sr + h * a.dout.sh;
      const char* o = a.out.p + b * a.out.sb + i * a.out.sr + h * a.out.sh;
      const char* ol = a.low.p ? a.low.p + b * a.low.sb + i * a.low.sr + h * a.low.sh : nullptr;
      for (int c = lane; c < s.C; c += 16) {
        const float x = elem<T>(p, c);
        sq = __builtin_fmaf(x, x, sq);
        dot = __builtin_fmaf(x, elem<T>(o, c) + (ol ? elem<T>(ol, c) : 0.0f), dot);
      }
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) {
      sq += __shfl_xor(sq, d);
      dot += __shfl_xor(dot, d);
    }
    if (!keys && lane == 0) a.delta[b * a.st_sb + h * a.st_sh + i] = dot;
    norm = used ? __builtin_sqrtf(sq) : 0.0f;
  }
  if (a.norms) {
#pragma unroll
    for (int d = 16; d < 64; d <<= 1) norm = fmaxf(norm, __shfl_xor(norm, d));
    if ((threadIdx.x & 63) == 0 && norm > 0.0f) atomicMax(a.norms + keys, __builtin_bit_cast(uint32_t, norm));
  }
}

template <typename T, int DP, int NT, int NW, bool KV>
__global__ __launch_bounds__(64 * NW, 2) void k_attn_bwd(const AttnBwdArgs a) {
  constexpr int BR = attn_keys<DP>(), NC = DP / 32, NO = DP / 16, TILE = BR * DP * 2, COLS = 16 * NT * NW;
  __shared__ __align__(1024) char smem[4 * TILE];
  __shared__ __align__(16) float stat[2][2][BR];  // [stage][lse, delta][row]
  const AttnShape& s = a.s;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 15, g = lane >> 4;

  int tile, head, b;
  block_place(blockIdx.x, a.heads, tile, head);
  const int rows_all = KV ? s.N : s.M;
  if (s.packed) {
    const int slot = KV ? tile : a.tiles - 1 - tile;
    b = packed_tile(KV ? s.k_index : s.q_index, s.B, rows_all, 1, COLS, slot, tile);
    if (b == kNoRow) {
      if (s.zero_rest & kRestOut) {
        const int part = slot - tile, parts = a.tiles - tile;
        const int32_t* index = KV ? s.k_index : s.q_index;
        const int end = s.B > 0 ? clampi(index[s.B], 0, rows_all) : 0;
        if (KV) {
          if (a.dk.p) zero_rows(a.dk, 0, head, s.D, end, rows_all, part, parts);
          if (a.dv.p) zero_rows(a.dv, 0, head, s.C, end, rows_all, part, parts);
        } else {
          zero_rows(a.dq, 0, head, s.D, end, rows_all, part, parts);
        }
      }
      return;
    }
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
  uint4 uo[NT][NC], wo[NT][NC];
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
        wo[n][c] = column_operand<T>(w, W.vec, s.C, c, 0);
      }
      if (!KV) {
        const int64_t i = b * a.st_sb + head * a.st_sh + c0 + at;
        clse[n] = a.lse[i] * kLog2e;
        cdelta[n] = a.delta[i];
      }
    }
  }
  int r_lo = 0, r_hi = 0, w_lo = 0, w_hi = 0, in_lo = 0, in_hi = 0;
  if (cn > 0 && t0 < cn) {
    int x;
    range(t0, r_lo, x);
    range(min(t0 + COLS, cn) - 1, x, r_hi);
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
  const int ds_e = scaled<T>() ? ds_exponent(a.norms) : 0;
  const float ds_up = __builtin_ldexpf(1.0f, ds_e);

  const TileLane<DP> ln;
  // the stream: tiles of rows [r_lo, r_hi), once for every query head (KV)
  const int heads = KV ? s.G : 1, h0 = KV ? head * s.G : head / s.G;
  const int steps = r_hi > r_lo ? (r_hi - r_lo + BR - 1) / BR : 0;
  auto issue = [&](int h, int row0, int stage) {
    char* t = smem + stage * 2 * TILE;
    const char* xb = X.p + b * X.sb + (int64_t)x0 * X.sr + (h0 + h) * X.sh;
    const char* yb = Y.p + b * Y.sb + (int64_t)x0 * Y.sr + (h0 + h) * Y.sh;
    load_tile<DP, BR, 64 * NW>(t, s.D, X.vec, [&](int r) { return xb + (int64_t)min(row0 + r, rn - 1) * X.sr; });
    load_tile<DP, BR, 64 * NW>(t + TILE, s.C, Y.vec,
                               [&](int r) { return yb + (int64_t)min(row0 + r, rn - 1) * Y.sr; });
    if (KV && tid < BR) {
      const int64_t i = b * a.st_sb + (h0 + h) * a.st_sh + x0 + min(row0 + tid, rn - 1);
      stat[stage][0][tid] = a.lse[i] * kLog2e;
      stat[stage][1][tid] = a.delta[i];
    }
  };
  if (s.D < DP || s.C < DP) {
    clear_tiles<64 * NW>(smem, 4 * TILE);
    __syncthreads();
  }
  if (steps > 0) issue(0, r_lo, 0);
  int stage = 0;
  for (int h = 0; h < heads; ++h)
    for (int st = 0; st < steps; ++st, stage ^= 1) {
      tile_barrier();
      if (st + 1 < steps)
        issue(h, r_lo + (st + 1) * BR, stage ^ 1);
      else if (h + 1 < heads)
        issue(h + 1, r_lo, stage ^ 1);
      const int row0 = r_lo + st * BR;
      if (row0 >= w_hi || row0 + BR <= w_lo) continue;
      const char* xt = smem + stage * 2 * TILE;
      const char* yt = xt + TILE;
      const bool masked = row0 + BR > in_hi || row0 < in_lo;
#pragma unroll
      for (int hf = 0; hf < BR / 32; ++hf) {
        uint4 pw[NT], dsw[NT];
        floatx4 sc[2][NT], dp[2][NT];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int n = 0; n < NT; ++n) sc[t][n] = dp[t][n] = floatx4{0, 0, 0, 0};
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            const uint4 xo = row_operand<DP>(xt, ln, 2 * hf + t, c);
            const uint4 yo = row_operand<DP>(yt, ln, 2 * hf + t, c);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              sc[t][n] = mfma_qk<T>(xo, uo[n][c], sc[t][n]);
              dp[t][n] = mfma_qk<T>(yo, wo[n][c], dp[t][n]);
            }
          }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          floatx4 rl{0, 0, 0, 0}, rd{0, 0, 0, 0};
          if (KV) {
            rl = *reinterpret_cast<const floatx4*>(&stat[stage][0][32 * hf + 16 * t + 4 * g]);
            rd = *reinterpret_cast<const floatx4*>(&stat[stage][1][32 * hf + 16 * t + 4 * g]);
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[t][n][r], a.c, -(KV ? rl[r] : clse[n])));
              float d = p * (dp[t][n][r] - (KV ? rd[r] : cdelta[n]));
              if (masked) {
                const int j = row0 + 32 * hf + 16 * t + 4 * g + r;
                const bool in = j >= lo[n] && j < hi[n];
                p = in ? p : 0.0f;
                d = in ? d : 0.0f;
              }
              // the weights and dS are rounded to the inputs' type for the matrix cores
              sc[t][n][r] = scaled<T>() ? p * (float)(1 << kWeightShift) : p;
              dp[t][n][r] = scaled<T>() ? d * ds_up : d;
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          pw[n] = uint4{pack2<T>(sc[0][n][0], sc[0][n][1]), pack2<T>(sc[0][n][2], sc[0][n][3]),
                        pack2<T>(sc[1][n][0], sc[1][n][1]), pack2<T>(sc[1][n][2], sc[1][n][3])};
          dsw[n] = uint4{pack2<T>(dp[0][n][0], dp[0][n][1]), pack2<T>(dp[0][n][2], dp[0][n][3]),
                         pack2<T>(dp[1][n][0], dp[1][n][1]), pack2<T>(dp[1][n][2], dp[1][n][3])};
        }
        if constexpr (KV) contract<T, DP, false, NO, NT>(yt, ln, hf, pw, dw, masked);
        contract<T, DP, true, NO, NT>(xt, ln, hf, dsw, du, masked);
      }
    }

  const float u_scale = s.scale * __builtin_ldexpf(1.0f, -ds_e);
  const float w_scale = scaled<T>() ? 1.0f / (1 << kWeightShift) : 1.0f;
  const AttnArray& DU = KV ? a.dk : a.dq;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int at = wc0 + 16 * n + col;
    if (at >= limit || (at >= cn && !(s.zero_rest & kRestOut))) continue;
    const bool none = at >= cn;
    if (DU.p) {
      char* p = DU.p + b * DU.sb + (int64_t)(c0 + at) * DU.sr + head * DU.sh;
#pragma unroll
      for (int ct = 0; ct < NO; ++ct) {
        floatx4 y = du[ct][n] * u_scale;
        if (none) y = floatx4{0, 0, 0, 0};
        store4<T>(p, 16 * ct + 4 * g, s.D, DU.vec, y[0], y[1], y[2], y[3]);
      }
    }
    if (KV && a.dv.p) {
      char* p = a.dv.p + b * a.dv.sb + (int64_t)(c0 + at) * a.dv.sr + head * a.dv.sh;
#pragma unroll
      for (int ct = 0; ct < NO; ++ct) {
        floatx4 y = dw[KV ? ct : 0][n] * w_scale;
        if (none) y = floatx4{0, 0, 0, 0};
        store4<T>(p, 16 * ct + 4 * g, s.C, a.dv.vec, y[0], y[1], y[2], y[3]);
      }
    }
  }
}

}  // namespace gs
