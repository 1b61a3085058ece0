// gs_attention.hip -- host side and kernel instances of softmax attention
// (include/gs_attention.h).
//
// Compiled as one unit (no GS_PART) or, in parallel, as GS_PARTS + 1 units: part 0
// is the host side and the kernels that do not depend on the dtype's width, parts
// 1 .. GS_PARTS one dtype and padded width each.
#include "gs_attention.h"

#include <algorithm>
#include <type_traits>

#include "gs_attn_bwd.h"
#include "gs_attn_fwd.h"

#define GS_PARTS 6
#ifndef GS_PART
#define GS_PART -1
#endif
#if GS_PART <= 0
#include "gs_attn_append.h"
#endif

namespace gs {

// Query tiles of 16 rows a wave owns (column tiles in the backward passes), per
// padded width: as many as its registers hold beside the operands in flight,
// since each operand read from LDS then feeds more matrix instructions (two
// waves a SIMD, 256 registers).  Forward of 8192 tokens, 32 heads, D = 128,
// causal: two tiles 617 us, three 572 us, four 2750 us (spilled); D = 256
// (2 x 2048 tokens, 8 heads): one 91 us, two 332 us (spilled).  dQ at D = 128: two
// 807 us, three 1947 us.  dK and dV at D = 128: two, with the operands of V in LDS
// (2 x 4096 tokens, 32 heads, no mask: 982 us; one tile 1248 us; two with all
// operands in registers spill).  Eight waves a workgroup instead of four: 4 to
// 10 % slower at every width.
constexpr int kAttnWaves = 4;
constexpr int attn_nq(int DP) { return DP == 256 ? 1 : DP == 128 ? 3 : 2; }
constexpr int attn_nt(int DP, bool KV) { return DP == 256 ? 1 : 2; }

// Few rows (k_attn_rows): one tile of 16 rows or four (DP = 256: one; four do not
// fit the registers), and as many waves as their rings fit in LDS.
constexpr int rows_waves(int DP) { return DP == 256 ? 2 : 4; }
constexpr int rows_most(int DP) { return DP == 256 ? 16 : 64; }

constexpr int attn_fwd_rows(int DP) { return 16 * kAttnWaves * attn_nq(DP); }
// and the smaller tile of short grids (DP = 256: none)
constexpr int attn_less_nq(int DP) { return DP == 256 ? 1 : attn_nq(DP) - 1; }
constexpr int attn_less_rows(int DP) { return 16 * kAttnWaves * attn_less_nq(DP); }
constexpr int attn_bwd_cols(int DP, bool KV) { return 16 * kAttnWaves * attn_nt(DP, KV); }

template <typename K, typename A>
hipError_t launch(K kernel, int64_t grid, int threads, const A& args, hipStream_t st) {
  void* p[1] = {const_cast<A*>(&args)};
  return hipLaunchKernel(reinterpret_cast<const void*>(kernel), dim3((unsigned)grid), dim3(threads), p, 0, st);
}

// rows: rows of a tile; few: k_attn_rows (16 or rows_most(DP)), else k_attn_fwd
// (attn_fwd_rows(DP) or, not over pages, attn_less_rows(DP))
template <typename T, int DP>
hipError_t attn_fwd(const AttnFwdArgs& a, bool paged, bool few, int rows, int64_t grid, hipStream_t st);
// cols: columns of a workgroup, attn_bwd_cols(DP, kv) or (not DP = 256) half of them
template <typename T, int DP>
hipError_t attn_bwd(const AttnBwdArgs& a, bool kv, int cols, int64_t grid, hipStream_t st);

#if GS_PART != 0
template <typename T, int DP, int NQ, bool PAGED>
hipError_t attn_rows(const AttnFwdArgs& a, int64_t grid, hipStream_t st) {
  constexpr int NW = rows_waves(DP);
  return launch(a.k.vec && a.v.vec ? &k_attn_rows<T, DP, NQ, NW, PAGED, true> : &k_attn_rows<T, DP, NQ, NW, PAGED, false>,
                grid, 64 * NW, a, st);
}
template <typename T, int DP, int NQ, bool PAGED>
hipError_t attn_tiles(const AttnFwdArgs& a, int64_t grid, hipStream_t st) {
  constexpr int NW = kAttnWaves;
  return launch(a.k.vec && a.v.vec ? &k_attn_fwd<T, DP, NQ, NW, PAGED, true> : &k_attn_fwd<T, DP, NQ, NW, PAGED, false>,
                grid, 64 * NW, a, st);
}
template <typename T, int DP>
hipError_t attn_fwd(const AttnFwdArgs& a, bool paged, bool few, int rows, int64_t grid, hipStream_t st) {
  hipError_t e;
  if (few) {
    constexpr int MOST = rows_most(DP) / 16;
    e = rows == 16 ? paged ? attn_rows<T, DP, 1, true>(a, grid, st) : attn_rows<T, DP, 1, false>(a, grid, st)
        : paged    ? attn_rows<T, DP, MOST, true>(a, grid, st)
                   : attn_rows<T, DP, MOST, false>(a, grid, st);
  } else {
    e = paged                        ? attn_tiles<T, DP, attn_nq(DP), true>(a, grid, st)
        : rows == attn_less_rows(DP) ? attn_tiles<T, DP, attn_less_nq(DP), false>(a, grid, st)
                                     : attn_tiles<T, DP, attn_nq(DP), false>(a, grid, st);
  }
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t units = (int64_t)(a.s.packed ? 1 : a.s.B) * a.s.M * a.s.Hq;
  return launch(&k_attn_join<T>, (units + 3) / 4, 256, a, st);
}
template <typename T, int DP, int NT, bool KV>
hipError_t attn_pass(const AttnBwdArgs& a, int64_t grid, hipStream_t st) {
  const bool wide = KV ? a.q.vec && a.dout.vec : a.k.vec && a.v.vec;
  return launch(wide ? &k_attn_bwd<T, DP, NT, kAttnWaves, KV, true> : &k_attn_bwd<T, DP, NT, kAttnWaves, KV, false>,
                grid, 64 * kAttnWaves, a, st);
}
template <typename T, int DP>
hipError_t attn_bwd(const AttnBwdArgs& a, bool kv, int cols, int64_t grid, hipStream_t st) {
  constexpr int LESS = DP == 256 ? attn_nt(DP, true) : 1;
  const bool less = cols < attn_bwd_cols(DP, kv);
  if (!kv)
    return less ? attn_pass<T, DP, LESS, false>(a, grid, st) : attn_pass<T, DP, attn_nt(DP, false), false>(a, grid, st);
  const hipError_t e =
      less ? attn_pass<T, DP, LESS, true>(a, grid, st) : attn_pass<T, DP, attn_nt(DP, true), true>(a, grid, st);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t units = (int64_t)(a.s.packed ? 1 : a.s.B) * a.s.N * a.s.Hkv;
  return launch(&k_attn_sum<T>, (units + 3) / 4, 256, a, st);
}
#define GS_ATTN_INSTANCE(T, DP)                                                               \
  template hipError_t attn_fwd<T, DP>(const AttnFwdArgs&, bool, bool, int, int64_t, hipStream_t); \
  template hipError_t attn_bwd<T, DP>(const AttnBwdArgs&, bool, int, int64_t, hipStream_t);
#if GS_PART == 1 || GS_PART == -1
GS_ATTN_INSTANCE(F16, 64)
#endif
#if GS_PART == 2 || GS_PART == -1
GS_ATTN_INSTANCE(F16, 128)
#endif
#if GS_PART == 3 || GS_PART == -1
GS_ATTN_INSTANCE(F16, 256)
#endif
#if GS_PART == 4 || GS_PART == -1
GS_ATTN_INSTANCE(BF16, 64)
#endif
#if GS_PART == 5 || GS_PART == -1
GS_ATTN_INSTANCE(BF16, 128)
#endif
#if GS_PART == 6 || GS_PART == -1
GS_ATTN_INSTANCE(BF16, 256)
#endif
#endif  // GS_PART != 0

#if GS_PART <= 0

namespace {

constexpr int64_t kMaxRows = (int64_t)1 << 30;
constexpr int64_t kMaxStride = (int64_t)1 << 44;
constexpr int64_t kMaxGrid = (1ll << 24) - 1;  // workgroups of 256 threads: below 2^32 threads

int padded_width(int64_t D, int64_t C) {
  const int64_t w = D > C ? D : C;
  return w <= 64 ? 64 : w <= 128 ? 128 : 256;
}

gs_status check(const gs_attention_problem* p) {
  if (!p) return GS_ERR_NULL_POINTER;
  if (p->B < 0 || p->B > (1 << 20) || p->M < 0 || p->M > kMaxRows || p->N < 0 || p->N > kMaxRows ||
      p->Hkv < 1 || p->Hq < p->Hkv || p->Hq > (1 << 14) || p->Hq % p->Hkv || p->D < 1 ||
      p->D > GAUSS_SUM_MAX_DIM || p->C < 1 || p->C > GAUSS_SUM_MAX_DIM || p->window < 0 ||
      p->window > kMaxRows || (p->window > 0 && !p->causal))
    return GS_ERR_BAD_SHAPE;
  if (p->dtype != GS_F16 && p->dtype != GS_BF16) return GS_ERR_UNSUPPORTED;
  const float c = p->scale * kLog2e;  // what the kernels use is finite as well
  if (!(c > -__builtin_inff()) || !(c < __builtin_inff())) return GS_ERR_BAD_TAU;
  return GS_SUCCESS;
}

AttnShape shape_of(const gs_attention_problem& p, const int32_t* q_index, const int32_t* k_index) {
  AttnShape s;
  s.q_index = q_index;
  s.k_index = k_index;
  s.B = (int32_t)p.B, s.M = (int32_t)p.M, s.N = (int32_t)p.N;
  s.Hq = (int32_t)p.Hq, s.Hkv = (int32_t)p.Hkv, s.G = (int32_t)(p.Hq / p.Hkv);
  s.D = (int32_t)p.D, s.C = (int32_t)p.C;
  s.packed = p.packed != 0, s.causal = p.causal != 0, s.zero_rest = p.zero_rest;
  s.window = (int32_t)p.window;
  s.scale = p.scale;
  return s;
}

// Address range [from, to) that an array's elements lie in.
struct Span {
  uintptr_t from = 0, to = 0;
  bool meets(const Span& o) const { return from < o.to && o.from < to; }
};

Span span_of(const void* p, int64_t bytes) {
  return {reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + (uintptr_t)(bytes > 0 ? bytes : 0)};
}

// Checks one array (B x rows x H x width, 16-bit elements) and brings it into the
// kernels' form.  An array without elements is not looked at.
gs_status array_of(const gs_attention_array* x, int64_t B, int64_t rows, int64_t H, int64_t width, bool output,
                   AttnArray& a, Span& span) {
  a = AttnArray{nullptr, 0, 0, 0, 0};
  span = Span{};
  if (B == 0 || rows == 0) return GS_SUCCESS;
  if (!x || !x->data) return GS_ERR_NULL_POINTER;
  if (reinterpret_cast<uintptr_t>(x->data) & 1) return GS_ERR_MISALIGNED;
  int64_t st[3] = {B > 1 ? x->batch_stride : 0, rows > 1 ? x->row_stride : 0, H > 1 ? x->head_stride : 0};
  int64_t n[3] = {B, rows, H};
  for (int64_t v : st)
    if (v < 0 || v > kMaxStride) return GS_ERR_BAD_SHAPE;
  __int128 last = width;
  for (int i = 0; i < 3; ++i) last += (__int128)(n[i] - 1) * st[i];
  if (last > ((__int128)1 << 60)) return GS_ERR_BAD_SHAPE;
  a.p = static_cast<char*>(x->data);
  a.sb = 2 * st[0], a.sr = 2 * st[1], a.sh = 2 * st[2];
  span = span_of(x->data, 2 * (int64_t)last);
  const int wide = output ? 4 : 8;  // elements of one access
  a.vec = a.sr < (1 << 24) && width % wide == 0 && (reinterpret_cast<uintptr_t>(x->data) & (2 * wide - 1)) == 0 &&
          st[0] % wide == 0 && st[1] % wide == 0 && st[2] % wide == 0;
  if (output) {  // distinct elements: dimensions by stride, each past all before it
    int64_t extent = width;
    for (int round = 0; round < 3; ++round) {
      int best = -1;
      for (int i = 0; i < 3; ++i)
        if (n[i] > 1 && (best < 0 || st[i] < st[best])) best = i;
      if (best < 0) break;
      if (st[best] < extent) return GS_ERR_ALIAS;
      extent += (n[best] - 1) * st[best];
      n[best] = 1;
    }
  }
  return GS_SUCCESS;
}

// |scale| log2 e, not below the smallest normal number: masked scores are -inf, and
// 0 * -inf is NaN (2^-126 times a score is 0 to every digit of the exponent).
float forward_factor(float scale) {
  const float c = (scale < 0 ? -scale : scale) * kLog2e;
  return c > 0x1p-126f ? c : 0x1p-126f;
}

// Tiles of one head: all sequences' (packed: as many as there can be, and one for
// the rows behind the last sequence) or one sequence's.
int64_t tiles_of(const gs_attention_problem& p, int64_t rows, int tile) {
  return p.packed ? rows / tile + p.B + 1 : (rows + tile - 1) / tile;
}

struct Carve {
  char* base;
  size_t off = 0;
  template <typename X>
  X* take(int64_t n) {
    X* r = base ? reinterpret_cast<X*>(base + off) : nullptr;
    off += ((size_t)n * sizeof(X) + 255) & ~(size_t)255;
    return r;
  }
};

// How a forward call is laid out: rows of a tile, query heads packed into the rows
// of a token, tiles and heads of the grid, parts of a row's keys, workspace.
struct FwdPlan {
  bool few;
  int rows;
  int64_t per, tiles, heads, splits, grid;
  float *part_o, *part_z;
  size_t total;
};

int64_t row_heads(const gs_attention_problem& p) { return (p.packed ? 1 : p.B) * p.M * p.Hq; }

// keys: of a sequence, at most (pages) or on average (packed).
FwdPlan fwd_plan(const gs_attention_problem& p, bool paged, int64_t keys, void* ws) {
  FwdPlan f{};
  const int DP = padded_width(p.D, p.C);
  const int64_t G = p.Hq / p.Hkv, B = p.packed ? 1 : p.B;
  // rows that share a key head: with the query heads of a token packed, keys and
  // values are read once for all of them.  The lengths of packed sequences lie on the
  // device, so their average decides, also for a long prompt among many single tokens.
  // Few rows against whole tiles, D = 128, causal: 64 single tokens over 2000 keys, 16
  // heads of each 216 and 223 us, 32 over 8 115 and 354 us; 64 x 16 tokens over 1000
  // keys, 32 over 8 89 and 199 us; but without shared heads 64 x 33 tokens 77 and 40 us,
  // 63 single tokens beside 1500 106 and 68 us (D = 64: 31 and 41 us)
  const int64_t shared = (p.packed && p.B > 0 ? (p.M + p.B - 1) / p.B : p.M) * G;
  const bool few = f.few = shared <= rows_most(DP);
  f.per = paged || few ? G : 1;
  f.rows = !few ? attn_fwd_rows(DP) : shared <= 16 ? 16 : rows_most(DP);
  f.tiles = tiles_of(p, p.M * f.per, f.rows);
  f.heads = (f.per > 1 || G == 1 ? p.Hkv : p.Hq) * B;
  // Short grids take a smaller tile: a workgroup is sooner done with each 64 keys and
  // the last round fuller.  D = 128, 192 rows -> 128, below two rounds of 512
  // workgroups: 1000 causal tokens, 16 heads 40 -> 32 us; 4 x 2048, no mask 158 -> 146
  // us; 8 packed sequences of 800 60 -> 56 us; 2 x 4096 causal 156 -> 159 us, and above
  // two rounds 192 rows are 8 % faster.  D = 64, 128 rows -> 64, where that fills the
  // GPU or the keys are too few to be cut: 4 x 512, 8 heads 16.1 -> 11.6 us; 2 x 2000
  // 46 -> 30 us; but 4000 tokens of 4 heads, cut in four, 39 -> 43 us.  Not over pages:
  // 2 chunks to 2048 tokens, 32 heads 156 -> 173 us.
  if (!few && !paged && DP != 256) {
    const int64_t less = tiles_of(p, p.M * f.per, attn_less_rows(DP)), full = f.tiles * f.heads;
    if (DP == 128 ? full < 1024 : full < 512 && (less * f.heads >= 512 || keys < 1024)) {
      f.rows = attn_less_rows(DP);
      f.tiles = less;
    }
  }
  // With fewer workgroups than two a CU a row's keys are cut into parts, none
  // shorter than 256 (512) keys.  Chunks over several long paged sequences, whose
  // lengths differ, take twice as many to even out; the parts cost the same for
  // short ones.  32 / 8 heads, D = 128, 512 -> 1024 workgroups: 4 chunks to 512 tokens
  // over 3000 to 12000 keys 405 -> 286 and 405 -> 269 us, where the longest chunk has
  // few tokens 272 -> 288 us; 8 to 256 over 2000 to 8000 276 -> 185 us; 2 to 2048 over
  // 1000 to 4000 156 -> 189 us.  D = 64: 8 to 300 over 1000 to 4000 60 -> 46 us.
  const bool uneven = paged && !few && p.B > 1 && keys >= 40 * DP;
  const int64_t wgs = f.tiles * f.heads, want = uneven ? 1024 : 512, least = few ? kLeastPart : 512;
  f.splits = wgs > 0 && keys >= 2 * least
                 ? std::max<int64_t>(1, std::min({want / wgs, keys / least, (int64_t)kMostParts}))
                 : 1;
  f.grid = wgs * f.splits;
  if (f.splits > 1) {
    Carve c{static_cast<char*>(ws)};
    f.part_o = c.take<float>(f.splits * row_heads(p) * p.C);
    f.part_z = c.take<float>(f.splits * row_heads(p) * 2);
    f.total = c.off;
  }
  return f;
}

int64_t dense_keys(const gs_attention_problem& p) { return p.packed && p.B > 0 ? p.N / p.B : p.N; }
int64_t cache_keys(const gs_attention_cache& c) { return std::min(c.table_width * c.page_size, kMaxRows); }

void plan_args(const FwdPlan& f, const gs_attention_problem& p, AttnFwdArgs& a) {
  a.per = (int32_t)f.per, a.tiles = (int32_t)f.tiles, a.heads = (int32_t)f.heads;
  a.wgs = (int32_t)(f.tiles * f.heads);
  a.splits = (int32_t)f.splits, a.part_o = f.part_o, a.part_z = f.part_z;
  a.neg = p.scale < 0;
  a.c = forward_factor(p.scale);
}

// How a backward call is laid out: columns of a workgroup of the dK, dV pass, the
// grids of both passes, workgroups that share a key head's query heads, workspace.
struct BwdPlan {
  int q_cols, k_cols;
  int64_t q_tiles, q_heads, k_tiles, k_heads, splits;
  float *delta, *lse2, *part;
  int64_t part_width;
  size_t total;
};

BwdPlan bwd_plan(const gs_attention_problem& p, bool want_kv, void* ws) {
  BwdPlan f{};
  const int DP = padded_width(p.D, p.C);
  const int64_t B = p.packed ? 1 : p.B, G = p.Hq / p.Hkv;
  f.q_heads = p.Hq * B;
  f.q_cols = attn_bwd_cols(DP, false);
  f.q_tiles = tiles_of(p, p.M, f.q_cols);
  // dQ: tiles of half the columns where those of all leave less than two workgroups
  // a CU.  1000 causal tokens, 16 heads, D = 128 42 -> 30 us; 4000, 8 heads 132 -> 98 us;
  // 4 x 512, 8 heads, D = 64 22 -> 17 us; at 700 workgroups (6 packed to 2047) 74 -> 85 us
  if (DP != 256 && f.q_tiles * f.q_heads < 512) {
    f.q_cols /= 2;
    f.q_tiles = tiles_of(p, p.M, f.q_cols);
  }
  f.k_heads = p.Hkv * B;
  f.k_cols = attn_bwd_cols(DP, true);
  f.k_tiles = tiles_of(p, p.N, f.k_cols);
  // dK, dV: 512 workgroups fill the GPU (two a CU); with a causal mask, whose tiles
  // have unequal numbers of pairs, it takes 1024 to even out.  Where there are fewer
  // the query heads of a key head are shared by several workgroups, as far as they
  // go (causal: to 2048, since the sums cost a pass anyway), and then (not D = 256)
  // tiles of half the columns are taken.  8192 tokens, 32 heads over 8, causal: 512
  // workgroups 1531 us, 1024 half tiles 1380 us, heads shared by two 1237 us, by
  // four 1181 us; 4 x 4096 tokens (1024 workgroups): not shared 1156 us, by two
  // 1228 us.  Half tiles at D = 64: 2 x 2000 causal tokens, 8 heads 70 -> 52 us.
  const bool even = !p.causal || (p.window > 0 && 2 * p.window <= p.N) || (p.packed && p.B >= 4);
  const int64_t want = even ? 512 : 1024, wgs = f.k_tiles * f.k_heads;
  f.splits = 1;
  if (wgs < want)
    while (f.splits < G && wgs * f.splits < (even ? want : 2 * want)) {
      do ++f.splits;
      while (G % f.splits);
    }
  if (DP != 256 && f.k_tiles * f.k_heads * f.splits < want) {
    f.k_cols /= 2;
    f.k_tiles = tiles_of(p, p.N, f.k_cols);
  }
  Carve c{static_cast<char*>(ws)};
  f.delta = c.take<float>(row_heads(p));
  f.lse2 = c.take<float>(row_heads(p));
  f.part_width = 2 * ((std::max(p.D, p.C) + 3) / 4 * 4);
  if (want_kv && f.splits > 1) f.part = c.take<float>(f.splits * B * p.N * p.Hkv * f.part_width);
  f.total = c.off;
  return f;
}

gs_status check_workspace(const void* ws, size_t have, size_t need) {
  if (need == 0) return GS_SUCCESS;
  if (!ws || have < need) return GS_ERR_WORKSPACE;
  if (reinterpret_cast<uintptr_t>(ws) & 255) return GS_ERR_MISALIGNED;
  return GS_SUCCESS;
}

// Any of the outputs over any of the others.
bool overlaps(const Span* out, int outs, const Span* in, int ins) {
  for (int i = 0; i < outs; ++i) {
    for (int j = 0; j < ins; ++j)
      if (out[i].meets(in[j])) return true;
    for (int j = 0; j < i; ++j)
      if (out[i].meets(out[j])) return true;
  }
  return false;
}

Span index_span(const gs_attention_problem& p, const int32_t* x) {
  return x ? span_of(x, 4 * (p.B + (p.packed ? 1 : 0))) : Span{};
}

template <typename F>
hipError_t by_type(const gs_attention_problem& p, F f) {
  const int DP = padded_width(p.D, p.C);
  if (p.dtype == GS_F16) return DP == 64 ? f(F16{}, std::integral_constant<int, 64>{})
                              : DP == 128 ? f(F16{}, std::integral_constant<int, 128>{})
                                          : f(F16{}, std::integral_constant<int, 256>{});
  return DP == 64 ? f(BF16{}, std::integral_constant<int, 64>{})
       : DP == 128 ? f(BF16{}, std::integral_constant<int, 128>{})
                   : f(BF16{}, std::integral_constant<int, 256>{});
}

gs_status index_args(const gs_attention_problem& p, const int32_t* q_index, const int32_t* k_index) {
  if (p.packed && (!q_index || !k_index)) return GS_ERR_NULL_POINTER;
  if ((reinterpret_cast<uintptr_t>(q_index) | reinterpret_cast<uintptr_t>(k_index)) & 3) return GS_ERR_MISALIGNED;
  return GS_SUCCESS;
}

gs_status run_fwd(const gs_attention_problem* p, const gs_attention_array* q, const gs_attention_array* k,
                  const gs_attention_array* v, const int32_t* q_index, const int32_t* k_index,
                  const gs_attention_array* out, const gs_attention_array* low, float* lse, void* ws, size_t ws_bytes,
                  hipStream_t stream) {
  gs_status st = check(p);
  if (st != GS_SUCCESS) return st;
  if ((p->B == 0 && !p->packed) || p->M == 0) return GS_SUCCESS;
  if ((st = index_args(*p, q_index, k_index)) != GS_SUCCESS) return st;
  const int64_t B = p->packed ? 1 : p->B;
  const FwdPlan f = fwd_plan(*p, false, dense_keys(*p), ws);
  if (f.grid > kMaxGrid) return GS_ERR_BAD_SHAPE;
  if ((st = check_workspace(ws, ws_bytes, f.total)) != GS_SUCCESS) return st;
  AttnFwdArgs a{};
  Span in[5], o[4];
  o[3] = span_of(ws, (int64_t)f.total);
  if ((st = array_of(q, B, p->M, p->Hq, p->D, false, a.q, in[0])) != GS_SUCCESS ||
      (low && (st = array_of(low, B, p->M, p->Hq, p->C, true, a.low, o[2])) != GS_SUCCESS) ||
      (st = array_of(k, B, p->N, p->Hkv, p->D, false, a.k, in[1])) != GS_SUCCESS ||
      (st = array_of(v, B, p->N, p->Hkv, p->C, false, a.v, in[2])) != GS_SUCCESS ||
      (st = array_of(out, B, p->M, p->Hq, p->C, true, a.out, o[0])) != GS_SUCCESS)
    return st;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return GS_ERR_MISALIGNED;
  if (lse) o[1] = span_of(lse, 4 * row_heads(*p));
  in[3] = index_span(*p, q_index), in[4] = index_span(*p, k_index);
  if (overlaps(o, 4, in, 5)) return GS_ERR_ALIAS;

  a.s = shape_of(*p, q_index, k_index);
  a.lse = lse;
  a.lse_sb = p->packed ? 0 : p->Hq * p->M;
  a.lse_sh = p->M;
  plan_args(f, *p, a);
  const hipError_t e = by_type(*p, [&](auto t, auto dp) {
    return attn_fwd<decltype(t), decltype(dp)::value>(a, false, f.few, f.rows, f.grid, stream);
  });
  return e == hipSuccess ? GS_SUCCESS : GS_ERR_HIP;
}

gs_status run_bwd(const gs_attention_problem* p, const gs_attention_array* q, const gs_attention_array* k,
                  const gs_attention_array* v, const int32_t* q_index, const int32_t* k_index,
                  const gs_attention_array* out, const gs_attention_array* low, const float* lse,
                  const gs_attention_array* dout,
                  const gs_attention_array* dq, const gs_attention_array* dk, const gs_attention_array* dv, void* ws,
                  size_t ws_bytes, hipStream_t stream) {
  gs_status st = check(p);
  if (st != GS_SUCCESS) return st;
  if (!dq && !dk && !dv) return GS_ERR_NULL_POINTER;
  if ((p->B == 0 && !p->packed) || (p->M == 0 && p->N == 0)) return GS_SUCCESS;
  if ((st = index_args(*p, q_index, k_index)) != GS_SUCCESS) return st;
  const int64_t B = p->packed ? 1 : p->B;
  const BwdPlan w = bwd_plan(*p, dk || dv, ws);
  if (w.q_tiles * w.q_heads > kMaxGrid || w.k_tiles * w.k_heads * w.splits > kMaxGrid) return GS_ERR_BAD_SHAPE;
  AttnBwdArgs a{};
  AttnArray ao, alow{};
  Span in[9], o[4];
  if ((st = array_of(q, B, p->M, p->Hq, p->D, false, a.q, in[0])) != GS_SUCCESS ||
      (st = array_of(k, B, p->N, p->Hkv, p->D, false, a.k, in[1])) != GS_SUCCESS ||
      (st = array_of(v, B, p->N, p->Hkv, p->C, false, a.v, in[2])) != GS_SUCCESS ||
      (st = array_of(out, B, p->M, p->Hq, p->C, false, ao, in[3])) != GS_SUCCESS ||
      (low && (st = array_of(low, B, p->M, p->Hq, p->C, false, alow, in[8])) != GS_SUCCESS) ||
      (st = array_of(dout, B, p->M, p->Hq, p->C, false, a.dout, in[4])) != GS_SUCCESS ||
      (dq && (st = array_of(dq, B, p->M, p->Hq, p->D, true, a.dq, o[0])) != GS_SUCCESS) ||
      (dk && (st = array_of(dk, B, p->N, p->Hkv, p->D, true, a.dk, o[1])) != GS_SUCCESS) ||
      (dv && (st = array_of(dv, B, p->N, p->Hkv, p->C, true, a.dv, o[2])) != GS_SUCCESS))
    return st;
  if (p->M > 0 && !lse) return GS_ERR_NULL_POINTER;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return GS_ERR_MISALIGNED;
  if (lse) in[5] = span_of(lse, 4 * row_heads(*p));
  in[6] = index_span(*p, q_index), in[7] = index_span(*p, k_index);
  if ((st = check_workspace(ws, ws_bytes, w.total)) != GS_SUCCESS) return st;
  o[3] = span_of(ws, (int64_t)w.total);
  if (overlaps(o, 4, in, 9)) return GS_ERR_ALIAS;

  a.s = shape_of(*p, q_index, k_index);
  a.lse2 = w.lse2;
  a.delta = w.delta;
  a.st_sb = p->packed ? 0 : p->Hq * p->M;
  a.st_sh = p->M;
  a.c = p->scale * kLog2e;

  AttnPrepArgs pr{};
  pr.s = a.s;
  pr.out = ao, pr.low = alow, pr.dout = a.dout;
  pr.lse = lse;
  pr.lse2 = w.lse2;
  pr.delta = w.delta;
  pr.st_sb = a.st_sb, pr.st_sh = a.st_sh;
  pr.units = row_heads(*p);

  hipError_t e = hipSuccess;
  // enough workgroups to fill the GPU several times
  const int64_t blocks = std::min<int64_t>(2048, (pr.units + 15) / 16);
  if (blocks > 0)
    e = p->dtype == GS_F16 ? launch(&k_attn_prep<F16>, blocks, 256, pr, stream)
                           : launch(&k_attn_prep<BF16>, blocks, 256, pr, stream);
  if (e != hipSuccess) return GS_ERR_HIP;
  for (int kv = 0; kv < 2; ++kv) {
    if (kv ? (!dk && !dv) || p->N == 0 : !dq || p->M == 0) continue;
    a.tiles = (int32_t)(kv ? w.k_tiles : w.q_tiles);
    a.heads = (int32_t)(kv ? w.k_heads : w.q_heads);
    a.splits = kv ? (int32_t)w.splits : 1;
    a.wgs = a.tiles * a.heads;
    a.part = w.part, a.part_width = (int32_t)w.part_width;
    e = by_type(*p, [&](auto t, auto dp) {
      return attn_bwd<decltype(t), decltype(dp)::value>(a, kv != 0, kv ? w.k_cols : w.q_cols, (int64_t)a.wgs * a.splits, stream);
    });
    if (e != hipSuccess) return GS_ERR_HIP;
  }
  return GS_SUCCESS;
}

// The pages of a cache.
gs_status cache_of(const gs_attention_problem& p, const gs_attention_cache* c, bool output, AttnArray& k, AttnArray& v,
                   AttnPages& pg, Span& ks, Span& vs) {
  if (!c) return GS_ERR_NULL_POINTER;
  if (c->pages < 0 || c->pages > kMaxRows || c->page_size < 1 || c->page_size > kMaxRows || c->table_width < 0 ||
      c->table_width > kMaxRows || (c->table_width > 0 && c->page_size > kMaxRows / c->table_width))
    return GS_ERR_BAD_SHAPE;
  if (p.B > 0 && (!c->lens || (c->table_width > 0 && !c->table))) return GS_ERR_NULL_POINTER;
  if ((reinterpret_cast<uintptr_t>(c->lens) | reinterpret_cast<uintptr_t>(c->table)) & 3) return GS_ERR_MISALIGNED;
  gs_status st = array_of(&c->k, c->pages, c->page_size, p.Hkv, p.D, output, k, ks);
  if (st == GS_SUCCESS) st = array_of(&c->v, c->pages, c->page_size, p.Hkv, p.C, output, v, vs);
  if (st != GS_SUCCESS) return st;
  if (output && c->pages > 0) {  // pages are written in 16-byte pieces
    const gs_attention_array* x[2] = {&c->k, &c->v};
    AttnArray* y[2] = {&k, &v};
    for (int i = 0; i < 2; ++i) {
      AttnArray in;
      Span s;
      if ((st = array_of(x[i], c->pages, c->page_size, p.Hkv, i ? p.C : p.D, false, in, s)) != GS_SUCCESS) return st;
      y[i]->vec = in.vec;
    }
  }
  pg.table = c->table;
  pg.lens = c->lens;
  pg.page_stride_k = k.sb, pg.page_stride_v = v.sb;
  pg.width = (int32_t)c->table_width, pg.pages = (int32_t)c->pages, pg.size = (int32_t)c->page_size;
  pg.shift = (c->page_size & (c->page_size - 1)) ? -1 : __builtin_ctzll((unsigned long long)c->page_size);
  return GS_SUCCESS;
}

gs_status run_paged(const gs_attention_problem* p, const gs_attention_array* q, const gs_attention_cache* cache,
                    const int32_t* q_index, const gs_attention_array* out, float* lse, void* ws, size_t ws_bytes,
                    hipStream_t stream) {
  gs_status st = check(p);
  if (st != GS_SUCCESS) return st;
  if (!p->causal) return GS_ERR_UNSUPPORTED;
  if ((p->B == 0 && !p->packed) || p->M == 0) return GS_SUCCESS;
  if (p->packed ? !q_index : q_index != nullptr) return p->packed ? GS_ERR_NULL_POINTER : GS_ERR_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(q_index) & 3) return GS_ERR_MISALIGNED;
  const int64_t B = p->packed ? 1 : p->B, G = p->Hq / p->Hkv;
  AttnFwdArgs a{};
  Span in[6], o[3];
  if ((st = array_of(q, B, p->M, p->Hq, p->D, false, a.q, in[0])) != GS_SUCCESS ||
      (st = cache_of(*p, cache, false, a.k, a.v, a.pg, in[1], in[2])) != GS_SUCCESS ||
      (st = array_of(out, B, p->M, p->Hq, p->C, true, a.out, o[0])) != GS_SUCCESS)
    return st;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return GS_ERR_MISALIGNED;
  if (lse) o[1] = span_of(lse, 4 * row_heads(*p));
  in[3] = index_span(*p, q_index);
  in[4] = span_of(cache->lens, 4 * p->B);
  in[5] = span_of(cache->table, 4 * p->B * cache->table_width);
  if (p->M * G > kMaxRows) return GS_ERR_BAD_SHAPE;
  const FwdPlan f = fwd_plan(*p, true, cache_keys(*cache), ws);
  if (f.grid > kMaxGrid) return GS_ERR_BAD_SHAPE;
  if ((st = check_workspace(ws, ws_bytes, f.total)) != GS_SUCCESS) return st;
  o[2] = span_of(ws, (int64_t)f.total);
  if (overlaps(o, 3, in, 6)) return GS_ERR_ALIAS;

  a.s = shape_of(*p, q_index, nullptr);
  a.lse = lse;
  a.lse_sb = p->packed ? 0 : p->M;
  a.lse_sh = p->M * B;
  plan_args(f, *p, a);
  const hipError_t e = by_type(*p, [&](auto t, auto dp) {
    return attn_fwd<decltype(t), decltype(dp)::value>(a, true, f.few, f.rows, f.grid, stream);
  });
  return e == hipSuccess ? GS_SUCCESS : GS_ERR_HIP;
}

gs_status run_append(const gs_attention_problem* p, const gs_attention_array* k, const gs_attention_array* v,
                     const gs_attention_cache* cache, const int32_t* q_index, hipStream_t stream) {
  gs_status st = check(p);
  if (st != GS_SUCCESS) return st;
  if (p->B == 0 || p->M == 0) return GS_SUCCESS;
  if (p->packed ? !q_index : q_index != nullptr) return p->packed ? GS_ERR_NULL_POINTER : GS_ERR_UNSUPPORTED;
  if (reinterpret_cast<uintptr_t>(q_index) & 3) return GS_ERR_MISALIGNED;
  const int64_t B = p->packed ? 1 : p->B;
  AttnAppendArgs a{};
  Span in[5], o[2];
  if ((st = array_of(k, B, p->M, p->Hkv, p->D, false, a.k, in[0])) != GS_SUCCESS ||
      (st = array_of(v, B, p->M, p->Hkv, p->C, false, a.v, in[1])) != GS_SUCCESS ||
      (st = cache_of(*p, cache, true, a.kp, a.vp, a.pg, o[0], o[1])) != GS_SUCCESS)
    return st;
  in[2] = index_span(*p, q_index);
  in[3] = span_of(cache->lens, 4 * p->B);
  in[4] = span_of(cache->table, 4 * p->B * cache->table_width);
  // keys and values may be interleaved in one allocation, but not the same
  if (overlaps(o, 1, in, 5) || overlaps(o + 1, 1, in, 5) || (cache->pages > 0 && a.kp.p == a.vp.p)) return GS_ERR_ALIAS;
  if (cache->table_width == 0 || cache->pages == 0) return GS_SUCCESS;
  a.s = shape_of(*p, q_index, nullptr);
  a.chunks = (int32_t)(((p->D > p->C ? p->D : p->C) + 7) / 8);
  const int64_t grid = (B * p->M + 3) / 4;
  if (grid > kMaxGrid) return GS_ERR_BAD_SHAPE;
  return launch(&k_attn_append, grid, 256, a, stream) == hipSuccess ? GS_SUCCESS : GS_ERR_HIP;
}

}  // namespace
#endif  // GS_PART <= 0
}  // namespace gs

#if GS_PART <= 0
extern "C" {

size_t gs_attention_fwd_workspace_size(const gs_attention_problem* p) {
  if (gs::check(p) != GS_SUCCESS || (p->B == 0 && !p->packed) || p->M == 0) return 0;
  return gs::fwd_plan(*p, false, gs::dense_keys(*p), nullptr).total;
}

gs_status gs_attention_fwd(const gs_attention_problem* p, const gs_attention_array* q, const gs_attention_array* k,
                           const gs_attention_array* v, const int32_t* q_index, const int32_t* k_index,
                           const gs_attention_array* out, const gs_attention_array* low, float* lse,
                           void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return gs::run_fwd(p, q, k, v, q_index, k_index, out, low, lse, workspace, workspace_bytes, stream);
}

size_t gs_attention_bwd_workspace_size(const gs_attention_problem* p, int want_dq, int want_dk, int want_dv) {
  if (gs::check(p) != GS_SUCCESS || (!want_dq && !want_dk && !want_dv)) return 0;
  return gs::bwd_plan(*p, want_dk || want_dv, nullptr).total;
}

gs_status gs_attention_bwd(const gs_attention_problem* p, const gs_attention_array* q, const gs_attention_array* k,
                           const gs_attention_array* v, const int32_t* q_index, const int32_t* k_index,
                           const gs_attention_array* out, const gs_attention_array* low, const float* lse,
                           const gs_attention_array* dout, const gs_attention_array* dq,
                           const gs_attention_array* dk, const gs_attention_array* dv, void* workspace,
                           size_t workspace_bytes, hipStream_t stream) {
  return gs::run_bwd(p, q, k, v, q_index, k_index, out, low, lse, dout, dq, dk, dv, workspace, workspace_bytes, stream);
}

size_t gs_attention_paged_workspace_size(const gs_attention_problem* p, const gs_attention_cache* cache) {
  if (gs::check(p) != GS_SUCCESS || !cache || (p->B == 0 && !p->packed) || p->M == 0 || cache->table_width < 0 ||
      cache->page_size < 1 || cache->page_size > gs::kMaxRows || cache->table_width > gs::kMaxRows)
    return 0;
  return gs::fwd_plan(*p, true, gs::cache_keys(*cache), nullptr).total;
}

gs_status gs_attention_paged(const gs_attention_problem* p, const gs_attention_array* q,
                             const gs_attention_cache* cache, const int32_t* q_index, const gs_attention_array* out,
                             float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return gs::run_paged(p, q, cache, q_index, out, lse, workspace, workspace_bytes, stream);
}

gs_status gs_attention_append(const gs_attention_problem* p, const gs_attention_array* k,
                              const gs_attention_array* v, const gs_attention_cache* cache, const int32_t* q_index,
                              hipStream_t stream) {
  return gs::run_append(p, k, v, cache, q_index, stream);
}

}  // extern "C"
#endif  // GS_PART <= 0
