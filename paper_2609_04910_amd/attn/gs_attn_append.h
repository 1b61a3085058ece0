// gs_attn_append.h -- keys and values of new tokens written to their places in the
// pages of a cache: token i of the qn new ones of a sequence of length L (new
// ones included) goes to position L - qn + i.  Bound by memory traffic: a wave
// takes a token, looks its place up once in scalar registers, and moves 16 bytes a
// lane (or single elements where rows are not 16-byte aligned).
#pragma once

#include "gs_attn_fwd.h"

namespace gs {

struct AttnAppendArgs {
  AttnShape s;           // M: rows of a sequence (dense) or of all (packed)
  AttnArray k, v;        // new tokens: row stride sr, head stride sh
  AttnArray kp, vp;      // pages: row stride sr, head stride sh
  AttnPages pg;
  int32_t chunks;        // 16-byte chunks of the wider of a row of K and one of V
};

__device__ __forceinline__ void move_chunk(const AttnArray& src, const AttnArray& dst, const char* from, char* to,
                                           int c, int width) {
  if (src.vec && dst.vec) {
    if (c * 8 < width) reinterpret_cast<uint4*>(to)[c] = reinterpret_cast<const uint4*>(from)[c];
    return;
  }
  for (int e = c * 8; e < min(c * 8 + 8, width); ++e)
    reinterpret_cast<uint16_t*>(to)[e] = reinterpret_cast<const uint16_t*>(from)[e];
}

__global__ __launch_bounds__(256) void k_attn_append(const AttnAppendArgs a) {
  const AttnShape& s = a.s;
  const int lane = threadIdx.x & 63;
  const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // over all sequences
  if (row >= (int64_t)(s.packed ? 1 : s.B) * s.M) return;
  int b, i, qn;
  if (s.packed) {
    int l = 0, r = s.B;  // the last sequence that starts at or before the row
    while (r - l > 1) {
      const int m = (l + r) >> 1;
      if (s.q_index[m] <= row)
        l = m;
      else
        r = m;
    }
    b = l;
    int first;
    seq_side(s.q_index, 1, b, s.M, first, qn);
    if (row < first || row >= first + qn) return;  // a row of no sequence
    i = (int)row - first;
  } else {
    b = (int)(row / s.M);
    i = (int)(row - (int64_t)b * s.M);
    qn = s.M;
  }
  const int64_t place = (int64_t)a.pg.lens[b] - qn + i;
  if (place < 0 || place >= (int64_t)a.pg.width * a.pg.size) return;
  const int64_t pi = place / a.pg.size, at = place - pi * a.pg.size;
  const int page = a.pg.table[(int64_t)b * a.pg.width + pi];
  if ((uint32_t)page >= (uint32_t)a.pg.pages) return;
  const int64_t sq = s.packed ? 0 : b, at_row = s.packed ? row : i;
  const char* k = a.k.p + sq * a.k.sb + at_row * a.k.sr;
  const char* v = a.v.p + sq * a.v.sb + at_row * a.v.sr;
  char* kp = a.kp.p + page * a.pg.page_stride_k + at * a.kp.sr;
  char* vp = a.vp.p + page * a.pg.page_stride_v + at * a.vp.sr;
  for (int j = lane; j < s.Hkv * a.chunks; j += 64) {
    const int h = j / a.chunks, c = j - h * a.chunks;
    move_chunk(a.k, a.kp, k + h * a.k.sh, kp + h * a.kp.sh, c, s.D);
    move_chunk(a.v, a.vp, v + h * a.v.sh, vp + h * a.vp.sh, c, s.C);
  }
}

}  // namespace gs
