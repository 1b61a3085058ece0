// gs_attn.h -- operand layouts and helpers shared by the softmax-attention
// kernels (gfx950 / CDNA4).
//
// As in the Gauss-sum kernels every contraction runs on the 16x16x32 matrix
// instruction in the transposed orientation: the rows of a streamed tile stand
// on the MFMA row index, the wave's own ("column") points on the lane index, so
// a lane holds 4 of the 16 rows of one column and the packed result of two row
// tiles is the B operand of the next contraction over those rows:
//     A operand: A[i = l%16][k = 8*(l/16) .. +7]
//     B operand: B[k = 8*(l/16) .. +7][j = l%16]
//     result   : D[i = 4*(l/16) + r][j = l%16]
// The contraction over 32 rows takes slot k = 8 g + z of lane group g = l/16 to
// row 16 (z / 4) + 4 g + z % 4, for which two transposing LDS reads give the
// A operand straight from the row-major tile.
//
// Tiles are copied from the caller's arrays to LDS without a register round trip
// (16 bytes a lane) where rows are 16-byte aligned and a multiple of 8 wide, and
// element by element otherwise.  A tile row is DP 16-bit elements (DP = 64, 128
// or 256, columns past the caller's width zero); its 16-byte chunk c lies at
// chunk c ^ swz(row), so that the operand reads spread over the LDS banks.
#pragma once

#include "../csrc/gs_common.h"

namespace gs {

constexpr int kNoRow = -1;
constexpr int kRestOut = 1, kRestLse = 2;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// One array of the caller: element (sequence b, row i, head h, column) at
// p + b*sb + i*sr + h*sh + 2*column (bytes; 4*column for 32-bit data).
struct AttnArray {
  char* p;
  int64_t sb, sr, sh;
  int32_t vec;  // rows 16-byte aligned and a multiple of 8 elements wide
};

// What every kernel of a call knows of it.
struct AttnShape {
  const int32_t* q_index;  // packed: B + 1 offsets; dense: B lengths or NULL
  const int32_t* k_index;
  int32_t B, M, N;         // dense: rows / keys of a sequence; packed: of all sequences together
  int32_t Hq, Hkv, G;      // G = Hq / Hkv
  int32_t D, C;
  int32_t packed, causal;
  int32_t zero_rest;       // rows of no sequence: kRestOut, kRestLse
  int32_t window;          // 0: none
  float scale;             // of the scores (natural units)
};

// One sequence: first row and count of its queries and keys.
struct AttnSeq {
  int32_t q0, qn, k0, kn;
};

__device__ __forceinline__ int clampi(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// First row and length of sequence b on one side (lengths and offsets are read
// as they are and brought into range, so no index leaves the arrays).
__device__ __forceinline__ void seq_side(const int32_t* index, int packed, int b, int rows, int& first, int& n) {
  if (packed) {
    first = clampi(index[b], 0, rows);
    n = clampi(index[b + 1], first, rows) - first;
  } else {
    first = 0;
    n = index ? clampi(index[b], 0, rows) : rows;
  }
}

__device__ __forceinline__ AttnSeq seq_of(const AttnShape& s, int b) {
  AttnSeq r;
  seq_side(s.q_index, s.packed, b, s.M, r.q0, r.qn);
  seq_side(s.k_index, s.packed, b, s.N, r.k0, r.kn);
  r.q0 = __builtin_amdgcn_readfirstlane(r.q0), r.qn = __builtin_amdgcn_readfirstlane(r.qn);
  r.k0 = __builtin_amdgcn_readfirstlane(r.k0), r.kn = __builtin_amdgcn_readfirstlane(r.kn);
  return r;
}

// For each lane its sequence's place by descending key (equal keys by number), B at
// most 64 sequences, one a lane.
__device__ __forceinline__ int place_by(int key, int B) {
  const int lane = threadIdx.x & 63;
  const int mine = lane < B ? clampi(key, 0, (1 << 25) - 1) << 6 | (63 - lane) : -1;
  int place = 0;
#pragma unroll 8
  for (int b = 0; b < B; ++b) place += __builtin_amdgcn_readlane(mine, b) > mine;
  return place;
}

// Tile `slot` of the packed rows: its sequence b, its index t within it and the
// sequence's number n of tiles (ceil(rows * per / tile)).  The tiles of all sequences
// are counted by one wave scan of the offsets, 64 sequences a step, up to 64
// sequences in descending order of `keys` (NULL: of their rows), so that the long
// ones start first.  Returns kNoRow where there is none, t then being the number of
// all tiles.
__device__ __forceinline__ int packed_tile(const int32_t* off, int B, int rows, int per, int tile, int slot,
                                           const int32_t* keys, int& t, int& n) {
  const int lane = threadIdx.x & 63;
  int base = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    int m = 0, seq = b0 + lane;
    if (seq < B) {
      const int e0 = clampi(off[seq], 0, rows);
      m = clampi(off[seq + 1], e0, rows) - e0;
      m = (int)(((int64_t)m * per + tile - 1) / tile);
    }
    if (B <= 64) {
      seq = __builtin_amdgcn_ds_permute(place_by(keys && lane < B ? keys[lane] : m, B) * 4, lane);
      m = __shfl(m, seq & 63);
      if (lane >= B) m = 0;
    }
    int end = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int x = __shfl_up(end, d);
      if (lane >= d) end += x;
    }
    const uint64_t hit = __ballot(slot - base < end);
    if (hit) {
      const int w = __builtin_ctzll(hit);
      n = __builtin_amdgcn_readlane(m, w);
      t = slot - base - (__builtin_amdgcn_readlane(end, w) - n);
      return __builtin_amdgcn_readlane(seq, w);
    }
    base += __builtin_amdgcn_readlane(end, 63);
  }
  t = base;
  return kNoRow;
}

// Streams and tiles of a launch: block id -> (tile, head).  Blocks go to the
// eight XCDs in turn, and each XCD has an L2 of its own: with a multiple of eight
// (sequence, head) streams every XCD gets a contiguous run of them, so the query
// heads that share a key head read its keys through one L2.
//
// The caller counts tiles from the one with most pairs.
__device__ __forceinline__ void block_place(int id, int heads, int& tile, int& head) {
  tile = id / heads;
  const int p = id - tile * heads;
  head = (heads & 7) == 0 ? (p & 7) * (heads >> 3) + (p >> 3) : p;
}

// Where two workgroups share a CU the first 256 blocks go to a CU each and the next
// 256 join them: those are turned round, eight by eight (so that each stays on its
// XCD), and the CU of the longest block gets the shortest of them.
__device__ __forceinline__ int folded(int id, int blocks) {
  const int groups = (min(blocks, 512) - 256) >> 3, g = (id - 256) >> 3;
  return id < 256 || g >= groups ? id : 256 + ((groups - 1 - g) << 3) + (id & 7);
}

// Rows that column point `at` (its index in its sequence) sees on the other
// side: [lo, hi).  ahead: place of the first query among the keys (keys - queries,
// or more where the keys end with a page table).  Queries see keys up to their own
// place (causal) and the last `window` of them; keys are seen the other way
// round.
__device__ __forceinline__ void query_range(const AttnShape& s, int at, int ahead, int kn, int& lo, int& hi) {
  lo = 0, hi = kn;
  if (s.causal) {
    const int end = at + ahead + 1;  // may be negative: nothing seen
    hi = clampi(end, 0, kn);
    if (s.window > 0 && end > s.window) lo = end - s.window;  // may lie past the keys: nothing seen
    lo = lo > hi ? hi : lo;
  }
}
__device__ __forceinline__ void key_range(const AttnShape& s, int at, int ahead, int qn, int& lo, int& hi) {
  lo = 0, hi = qn;
  if (s.causal) {
    const int64_t first = (int64_t)at - ahead;
    lo = first < 0 ? 0 : first > qn ? qn : (int)first;
    if (s.window > 0) {
      const int64_t end = first + s.window;
      hi = end < lo ? lo : end < qn ? (int)end : qn;
    }
  }
}

template <typename T>
__device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <>
__device__ __forceinline__ uint32_t pack2<F16>(float lo, float hi) {
  return pack_f16(lo, hi);
}
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
template <>
__device__ __forceinline__ uint32_t pack2<BF16>(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(floatx2{lo, hi}, bf16x2));
}

template <typename T>
constexpr uint32_t exponent_bits() {
  return sizeof(typename T::storage) == 2 && __is_same(T, F16) ? 0x7c00u : 0x7f80u;
}

// Whether any of the eight elements is an infinity or NaN.
template <typename T>
__device__ __forceinline__ bool not_finite(const uint4& a) {
  constexpr uint32_t e = exponent_bits<T>();
  bool bad = false;
  for (uint32_t x : {a.x, a.y, a.z, a.w}) bad |= (x & e) == e || ((x >> 16) & e) == e;
  return bad;
}

// ------------------------------------------------------------------ LDS tiles

typedef __attribute__((address_space(3))) char attn_lds;
__device__ __forceinline__ uint32_t lds_offset(const void* p) { return (uint32_t)(uintptr_t)(const attn_lds*)p; }

// 64 lanes x 16 (4) bytes from base + per-lane offset, or from per-lane
// addresses, to LDS bytes lds + 16 (4) * lane.  Assembly, so that the compiler does
// not count the copy: the tile loop waits (copies_done) before the barrier that
// publishes it.  The compiler's waits for its own loads take the copies in all the
// same: where operands loaded before a tile loop are first used inside it (the query
// operands of the forward kernels, the columns' of dK and dV where they are in
// registers), it waits there in every tile, and so for most or all of the next
// tile's copies.  The s_nop separates the write of m0 from its use.
__device__ __forceinline__ void copy16(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}
__device__ __forceinline__ void copy16(const char* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
               :
               : "s"(lds), "v"(src)
               : "memory", "m0");
}
__device__ __forceinline__ void copy4(const void* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
               :
               : "s"(lds), "v"(off), "s"(base)
               : "memory", "m0");
}

// Every copy of this wave has landed, and no LDS access of it is under way.
__device__ __forceinline__ void copies_done() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }

// The workgroup's barrier, with this wave's LDS writes done.
__device__ __forceinline__ void tile_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// The XOR of a row's chunks: the row reads (eight rows, one chunk) and the
// transposing reads (four rows, two chunks) spread over the banks.  (A swizzle
// that spreads 16 rows over 256 bytes measured the same, with more registers.)
__host__ __device__ constexpr int swz(int row) { return ((row & 3) << 1) | ((row >> 2) & 1); }

// A value that is the same in all lanes, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// This thread's share of a tile of ROWS rows of DP elements that THREADS threads
// copy: one 16-byte chunk of each of the rows row0 + i * STEP.  (The swizzle only
// moves bits, and row0 < STEP, so swz(row0 + i * STEP) = swz(row0) ^ swz(i * STEP).)
template <int DP, int ROWS, int THREADS>
struct TileCopy {
  static constexpr int NCH = DP / 8, STEP = THREADS / NCH, N = ROWS / STEP;
  static_assert(THREADS % NCH == 0 && ROWS % STEP == 0 && (STEP & (STEP - 1)) == 0, "whole rows");
  int tid, row0, chunk0;
  __device__ __forceinline__ explicit TileCopy(int t) : tid(t) {
    row0 = tid / NCH;
    chunk0 = (tid % NCH) ^ swz(row0);
  }
  __device__ __forceinline__ int chunk(int i) const { return chunk0 ^ swz(i * STEP); }
  // LDS bytes of this wave's share of step i
  __device__ __forceinline__ uint32_t lds(const char* tile, int i) const {
    return uniform(lds_offset(tile)) + i * THREADS * 16 + uniform(tid >> 6) * 1024;
  }

  // Rows first .. of an array (row `first` at base), none past row `last` of the
  // tile (that row is repeated: what is past the end is masked).  Rows 16-byte
  // aligned, a multiple of 8 wide, ROWS * sr below 2^31.  Every wave issues N
  // copies (each row of a wave's share has a lane with a column).
  __device__ __forceinline__ void wide(char* tile, const char* base, uint32_t sr, int last, int width) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (chunk(i) * 8 < width)
        copy16(base, (uint32_t)min(row0 + i * STEP, last) * sr + chunk(i) * 16, lds(tile, i));
  }
  // The same from row addresses: row(i) is that of the thread's i-th row.
  template <typename Row>
  __device__ __forceinline__ void wide_rows(char* tile, int width, Row row) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const char* src = row(i);
      if (chunk(i) * 8 < width) copy16(src + chunk(i) * 16, lds(tile, i));
    }
  }
  // The same where the RW rows of each of a wave's copies lie sr apart: base(i) is
  // the address, the same in all lanes, of the first row of the wave's copy i, the
  // tile's row wave_row + i * STEP.
  static constexpr int RW = 64 / NCH;
  __device__ __forceinline__ int wave_row() const { return uniform(tid >> 6) * RW; }
  template <typename Base>
  __device__ __forceinline__ void wide_bases(char* tile, int width, uint32_t sr, Base base) const {
    const uint32_t row = (uint32_t)((tid & 63) / NCH) * sr;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (chunk(i) * 8 < width) copy16(base(i), row + chunk(i) * 16, lds(tile, i));
  }
  // Element by element (any alignment and width).
  template <typename Row>
  __device__ __forceinline__ void narrow_rows(char* tile, int width, Row row) const {
#pragma unroll 1
    for (int i = 0; i < N; ++i) {
      const char* src = row(i);
      const int c = chunk(i) * 8;
      uint32_t x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = c + e < width ? reinterpret_cast<const uint16_t*>(src)[c + e] : 0u;
      *reinterpret_cast<uint4*>(tile + (i * THREADS + tid) * 16) =
          uint4{x[0] | x[1] << 16, x[2] | x[3] << 16, x[4] | x[5] << 16, x[6] | x[7] << 16};
    }
  }
};

// Zeros over all of a workgroup's tiles: the columns past the caller's width are
// not written by the copies.
template <int THREADS>
__device__ __forceinline__ void clear_tiles(char* tiles, int bytes) {
  for (int at = threadIdx.x * 16; at < bytes; at += THREADS * 16)
    *reinterpret_cast<uint4*>(tiles + at) = uint4{0, 0, 0, 0};
}

// The lane's places in a tile: row operands (row l%16, chunk 4c + l/16) and
// transposed operands (rows 4 (l/16) .. +3, columns 16 ct + 4 (l%4) .. +3).
template <int DP>
struct TileLane {
  int row[2];
  int tr[4];
  __device__ __forceinline__ TileLane() {
    const int l = threadIdx.x & 63, i = l & 15, g = l >> 4;
    for (int p = 0; p < 2; ++p) row[p] = i * DP * 2 + ((4 * p + g) ^ swz(i)) * 16;
    const int r = 4 * g + ((l >> 2) & 3);
    for (int p = 0; p < 4; ++p) tr[p] = r * DP * 2 + ((2 * p + ((l >> 1) & 1)) ^ swz(r)) * 16 + (l & 1) * 8;
  }
};

// Row operand: rows 16 t .. of the tile, columns 32 c .. .
template <int DP>
__device__ __forceinline__ uint4 row_operand(const char* tile, const TileLane<DP>& ln, int t, int c) {
  return *reinterpret_cast<const uint4*>(tile + ln.row[c & 1] + (c >> 1) * 128 + t * 16 * DP * 2);
}

typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4v lds_short4v;
__device__ __forceinline__ uint2 read_tr(const char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4v*)(attn_lds*)p));
}
// Transposed operand: columns 16 ct .. of the tile on the MFMA rows, its rows
// 32 s .. +31 contracted.
template <int DP>
__device__ __forceinline__ uint4 tr_operand(const char* tile, const TileLane<DP>& ln, int s, int ct) {
  const char* p = tile + ln.tr[ct & 3] + (ct >> 2) * 128 + s * 32 * DP * 2;
  const uint2 a = read_tr(p), b = read_tr(p + 16 * DP * 2);
  return uint4{a.x, a.y, b.x, b.y};
}

// No LDS access and no matrix instruction moves across (vector arithmetic may):
// keeps a stage's LDS reads one stage ahead of the
// matrix instructions that use them.  Left to itself the compiler issues a whole
// phase's reads at once, and holds them in registers that the sums need (the
// D = 128 kernels then spilled 50 to 450 values inside the tile loop).
__device__ __forceinline__ void stage_fence() { __builtin_amdgcn_sched_barrier(0x6); }

// N stages of a contraction: operand i is read P stages before use(i, operand), the
// first P of them before the first stage (preload), and the last stages read the
// first operands of what comes next (into `next`), so that no phase begins with a
// wait for LDS.  The loops unroll: i is a constant in load and use.
template <int P>
struct Ahead {
  uint4 x[P + 1];
  template <typename Load>
  __device__ __forceinline__ void preload(Load load) {
#pragma unroll
    for (int i = 0; i < P; ++i) x[i] = load(i);
  }
};
struct NoLoad {};
template <int N, int P, typename Load, typename Use, typename Next>
__device__ __forceinline__ void stages(Ahead<P>& ops, Load load, Use use, Ahead<P>& next, Next next_load) {
  static_assert(N >= P, "stages");
#pragma unroll
  for (int i = 0; i < N; ++i) {
    if (i + P < N)
      ops.x[(i + P) % (P + 1)] = load(i + P);
    else if constexpr (!__is_same(Next, NoLoad))
      next.x[i + P - N] = next_load(i + P - N);
    stage_fence();
    use(i, ops.x[i % (P + 1)]);
    stage_fence();
  }
}

// Tiles some of whose rows some columns do not see.  Their weights are zero
// there, but 0 * NaN is NaN: an infinity or NaN may reach only the columns that
// see its row.  So each thread zeroes such elements in the chunks of the tile that
// it copied itself, before the barrier that publishes the tile, and leaves the
// tile's number in `mark` where there were any; the columns that see those rows
// are then found apart (a rare path that keeps to a few registers).  Returns
// whether the thread found any.
template <typename T, int DP, int ROWS, int THREADS>
__device__ __forceinline__ bool clean_tile(char* tile, int tid) {
  constexpr uint32_t e = exponent_bits<T>();
  bool any = false;
#pragma unroll
  for (int it = 0; it < ROWS * DP / 8 / THREADS; ++it) {
    uint4* p = reinterpret_cast<uint4*>(tile + (it * THREADS + tid) * 16);
    const uint4 x = *p;
    if (not_finite<T>(x)) {
      auto fix = [](uint32_t y) {
        return ((y & e) == e ? 0u : y & 0xffffu) | (((y >> 16) & e) == e ? 0u : y & 0xffff0000u);
      };
      *p = uint4{fix(x.x), fix(x.y), fix(x.z), fix(x.w)};
      any = true;
    }
  }
  return any;
}

// ------------------------------------------------------------- 16-bit output

// Four neighbouring 32-bit sums of a row of `width`.
__device__ __forceinline__ void store_sums(float* row, int c, int width, const floatx4& x) {
  if ((width & 3) == 0) {
    if (c < width) *reinterpret_cast<floatx4*>(row + c) = x;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < width) row[c + e] = x[e];
  }
}
__device__ __forceinline__ floatx4 load_sums(const float* row, int c, int width) {
  floatx4 x{0, 0, 0, 0};
  if ((width & 3) == 0) {
    if (c < width) x = *reinterpret_cast<const floatx4*>(row + c);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (c + e < width) x[e] = row[c + e];
  }
  return x;
}

// Four neighbouring columns of one row, rounded to T once.
template <typename T>
__device__ __forceinline__ void store4(char* row, int c, int width, int vec, float x0, float x1, float x2,
                                       float x3) {
  const uint32_t a = pack2<T>(x0, x1), b = pack2<T>(x2, x3);
  uint16_t* p = reinterpret_cast<uint16_t*>(row) + c;
  if (vec) {
    if (c < width) *reinterpret_cast<uint2*>(p) = uint2{a, b};
  } else {
    if (c < width) p[0] = (uint16_t)a;
    if (c + 1 < width) p[1] = (uint16_t)(a >> 16);
    if (c + 2 < width) p[2] = (uint16_t)b;
    if (c + 3 < width) p[3] = (uint16_t)(b >> 16);
  }
}

// A row's result, which lies between its smallest and largest value: the weights'
// own rounding can bring it past fp16's largest number by up to 2^-11 of it, and from
// 2^-12 on it would round to infinity.
template <typename T>
__device__ __forceinline__ float between(float y) {
  constexpr float most = 65504.0f;
  return __is_same(T, F16) && __builtin_fabsf(y) < __builtin_inff() ? fminf(fmaxf(y, -most), most) : y;
}

// What rounding x to T leaves.
template <typename T>
__device__ __forceinline__ float left(float x) {
  return x - T::to_float((uint16_t)pack2<T>(x, 0.0f));
}

// Whether row i of packed rows belongs to a sequence (the offsets not decreasing).
__device__ __forceinline__ bool in_sequences(const int32_t* off, int B, int i) {
  return B > 0 && i >= off[0] && i < off[B];
}

// The rows of no sequence, before the first and behind the last, in turn.
struct RestRows {
  int lo, hi, n;
  __device__ __forceinline__ RestRows(const int32_t* off, int B, int rows) {
    lo = B > 0 ? clampi(off[0], 0, rows) : 0;
    hi = B > 0 ? clampi(off[B], lo, rows) : 0;
    n = lo + rows - hi;
  }
  __device__ __forceinline__ int64_t row(int i) const { return i < lo ? i : hi + (i - lo); }
};

// Zeros in rows part, part + parts, ... of them, of one head.
__device__ __forceinline__ void zero_rest_rows(const AttnArray& x, int head, int width, const RestRows& rest, int part,
                                               int parts) {
  for (int64_t i = part; i < rest.n; i += parts) {
    uint16_t* p = reinterpret_cast<uint16_t*>(x.p + rest.row((int)i) * x.sr + head * x.sh);
    for (int c = threadIdx.x; c < width; c += blockDim.x) p[c] = 0;
  }
}

}  // namespace gs
