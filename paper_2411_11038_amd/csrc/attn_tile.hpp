// Pieces that the attention kernels share: which keys a query sees, places of blocks in packed sequences, tiles of rows in LDS and the
// fragments of the matrix instructions that are read from them.
//
// All kernels use v_mfma_f32_32x32x16_bf16 or, for fp32, eight v_mfma_f32_32x32x2_f32 on the same fragments: a lane holds 8 of the 16
// contraction elements of one row (column) of an operand, elements 8 (lane / 32) .. + 7 of row (column) lane % 32.  The result has column
// lane % 32 and, in register i, row (i & 3) + 8 (i >> 2) + 4 (lane / 32).  Eight neighbouring registers of a result are thus a fragment
// of the next product's operand, if that product's other operand takes its 16 contraction elements in the same order (col_frag does):
// probabilities go from one product to the next without leaving their lane.
#pragma once
#include "gemm_epilogue.hpp"
#include "lds_copy.hpp"
#include "rows.hpp"

#include <initializer_list>

namespace efqat {

constexpr int64_t kAttnMostRows = INT64_C(1) << 28;          // sums of three such fit 32 bits

// token at position p sees key j (< keys of the sequence)
struct AttnMask {
  int causal, window, sinks;
  __device__ __forceinline__ bool sees(int p, int j) const {
    const int d = p - j;                             // no short cuts: no branch may lie between a product and what reads its result
    return ((causal == 0) | (d >= 0)) & ((window == 0) | ((d < window) & (-d < window)) | (j < sinks));
  }
  // all of p0 .. p1 see all of j0 .. j1
  __device__ __forceinline__ bool sees_all(int p0, int p1, int j0, int j1) const {
    return (!causal || j1 <= p0) && (!window || (p1 - j0 < window && j1 - p0 < window) || j1 < sinks);
  }
  // some of p0 .. p1 may see some of j0 .. j1
  __device__ __forceinline__ bool sees_some(int p0, int p1, int j0, int j1) const {
    return (!causal || j0 <= p1) && (!window || (p0 - j1 < window && j0 - p1 < window) || j0 < sinks);
  }
};

// Sequences packed into rows: sequence s is rows start[s] .. start[s + 1] - 1, or rows / n rows each (start NULL).  Offsets are data of the
// device: they are cut to the rows that exist.
struct Packed {
  const int32_t* start;
  int rows, n;
  __device__ __forceinline__ int2 place(int s) const {               // first row, rows
    if (!start) {
      const int each = rows / n;
      return make_int2(s * each, each);
    }
    int a = start[s], b = start[s + 1];
    a = a < 0 ? 0 : a > rows ? rows : a;
    b = b < a ? a : b > rows ? rows : b;
    return make_int2(a, b - a);
  }
  // at most so many tiles have rows
  __host__ int64_t most_tiles(int tile) const {
    return start ? ceil_div(rows, tile) + n - 1 : n * ceil_div(rows / n, tile);
  }
};
// Sequence and tile in it of tile number t of all sequences; false: there are not so many.  A wavefront looks at 64 sequences at a time.
__device__ __forceinline__ bool find_tile(const Packed& p, int tile_rows, int t, int* seq, int* tile) {
  if (!p.start) {
    const int each = (int)((p.rows / p.n + tile_rows - 1) / tile_rows);
    *seq = t / each;
    *tile = t - *seq * each;
    return true;
  }
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < p.n; base += 64) {
    int n = 0;
    if (base + lane < p.n) n = (p.place(base + lane).y + tile_rows - 1) / tile_rows;
    int end = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(end, o, 64);
      end += lane >= o ? v : 0;
    }
    const uint64_t past = __ballot(end > t);
    if (past) {
      const int l = __builtin_ctzll(past);
      *seq = base + l;
      *tile = t - __builtin_amdgcn_readlane(end - n, l);
      return true;
    }
    t -= __builtin_amdgcn_readlane(end, 63);
  }
  return false;
}

// ---- fragments
template <typename T>
struct Frag;
template <>
struct Frag<bf16_t> {
  bf16x8_t v;
};
template <>
struct Frag<float> {
  float v[8];
};
__device__ __forceinline__ void mma(const Frag<bf16_t>& a, const Frag<bf16_t>& b, floatx16_t& c) {
#if defined(__HIP_DEVICE_COMPILE__)
  c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a.v, b.v, c, 0, 0, 0);
#endif
}
__device__ __forceinline__ void mma(const Frag<float>& a, const Frag<float>& b, floatx16_t& c) {
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
  for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[e], b.v[e], c, 0, 0, 0);
#endif
}
// registers 8 s .. 8 s + 7 of a result as an operand; bf16: rounded to nearest even
template <typename T>
__device__ __forceinline__ Frag<T> frag_of(const floatx16_t& c, int s) {
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
    uint4 w;
    w.x = pack_bf16x2(c[8 * s], c[8 * s + 1]);
    w.y = pack_bf16x2(c[8 * s + 2], c[8 * s + 3]);
    w.z = pack_bf16x2(c[8 * s + 4], c[8 * s + 5]);
    w.w = pack_bf16x2(c[8 * s + 6], c[8 * s + 7]);
    f.v = __builtin_bit_cast(bf16x8_t, w);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) f.v[e] = c[8 * s + e];
  }
  return f;
}
// what the rounding of frag_of took, rounded itself: both together have 16 bits
__device__ __forceinline__ Frag<bf16_t> rest_of(const floatx16_t& c, int s, const Frag<bf16_t>& of) {
  const uint4 w = __builtin_bit_cast(uint4, of.v);
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
    y[i] = pack_bf16x2(c[8 * s + 2 * i] - __uint_as_float(x[i] << 16), c[8 * s + 2 * i + 1] - __uint_as_float(x[i] & 0xFFFF0000u));
  Frag<bf16_t> f;
  f.v = __builtin_bit_cast(bf16x8_t, make_uint4(y[0], y[1], y[2], y[3]));
  return f;
}
// made where this stands: the compiler may not move it behind a branch, nearer to where it is used
__device__ __forceinline__ void hold(float& v) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(v));
#endif
}
__device__ __forceinline__ void hold(Frag<bf16_t>& f) {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(f.v));
#endif
}
__device__ __forceinline__ void hold(Frag<float>& f) {
#pragma unroll
  for (int e = 0; e < 8; ++e) hold(f.v[e]);
}
__device__ __forceinline__ floatx16_t zero16() {
  floatx16_t z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.0f;
  return z;
}
// row of a result that register i holds in this lane
__device__ __forceinline__ int result_row(int i) { return (i & 3) + 8 * (i >> 2) + 4 * ((threadIdx.x >> 5) & 1); }
// first row of a result that this lane holds, made where this stands: rows made from it do not occupy registers elsewhere
__device__ __forceinline__ int row_here() {
  int r = 4 * ((threadIdx.x >> 5) & 1);
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("" : "+v"(r));
#endif
  return r;
}
__device__ __forceinline__ int row_of(int i) { return (i & 3) + 8 * (i >> 2); }

// 8 elements of a row of a matrix in memory as an operand, 16-byte aligned; not `ok`: zeros
template <typename T>
__device__ __forceinline__ Frag<T> load_frag(const T* p, bool ok) {
  Frag<T> f;
  if constexpr (sizeof(T) == 2) {
    uint4 w = make_uint4(0, 0, 0, 0);
    if (ok) w = *reinterpret_cast<const uint4*>(p);
    f.v = __builtin_bit_cast(bf16x8_t, w);
  } else {
    float4 a = make_float4(0, 0, 0, 0), b = a;
    if (ok) {
      a = *reinterpret_cast<const float4*>(p);
      b = *reinterpret_cast<const float4*>(p + 4);
    }
    f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
    f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
  }
  return f;
}

#if defined(__HIP_DEVICE_COMPILE__)
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char*)p; }
template <class V>
__device__ __forceinline__ V lds_read(uint32_t at) {
  return *(__attribute__((address_space(3))) const V*)(uintptr_t)at;
}
#endif

// ---- a tile of rows of DP (64, 96 or 128) features in LDS.  Its 16-byte pieces are swizzled by row so that both ways of reading it spread over the
// banks: neighbouring rows at the same piece (row_frag), and four rows at four neighbouring pieces (col_frag, bf16, transposing reads)
// or two rows four apart at eight neighbouring pieces (col_frag, fp32).
template <typename T, int DP>
struct RowTile {
  static constexpr int PITCH = DP <= 64 ? 64 : 128;                                  // features that a row has room for
  static constexpr int ROW = PITCH * (int)sizeof(T), CH = ROW / 16, RPI = 1024 / ROW;   // bytes and pieces of a row, rows of one copy
  static constexpr int KS = DP / 16, ND = DP / 32;                                   // contraction steps, result tiles of a row
  __device__ static __forceinline__ int swz(int row) {
    if constexpr (sizeof(T) == 4) return ((row >> 2) & 1) << 3 | ((row >> 3) & 1) << 2 | (row & 3);
    else if constexpr (PITCH == 128) return (row & 3) << 2 | ((row >> 2) & 3);
    else return ((row >> 1) & 1) << 2 | ((row >> 2) & 3);
  }
  // copy number `slot` of a tile: the rows slot * RPI .. + RPI - 1, those at `valid` and behind and pieces behind `pieces` as zeros
  __device__ static __forceinline__ void copy(const char* base, int64_t ld_bytes, int valid, int pieces, char* lds, int slot) {
    const int lane = threadIdx.x & 63;
    const int row = slot * RPI + lane / CH, piece = (lane % CH) ^ swz(row);
    const char* src = row < valid && piece < pieces ? base + row * ld_bytes + piece * 16 : zero_page();
    dma16(src, lds + slot * 1024);
  }
  // Addresses of pieces differ by exclusive ors with constants: tiles lie at multiples of a row, and so does everything that is added.
  // contraction step ks of row `row` (a multiple of 32) + lane % 32
  __device__ static __forceinline__ Frag<T> row_frag(const char* lds, int row, int ks) {
    Frag<T> f;
#if defined(__HIP_DEVICE_COMPILE__)
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const uint32_t base = lds_address(lds) + r * ROW + ((h ^ swz(r)) << 4);
      f.v = lds_read<bf16x8_t>((base ^ (ks << 5)) + row * ROW);
    } else {
      const uint32_t base = lds_address(lds) + r * ROW + (((2 * h) ^ swz(r)) << 4);
      const float4 a = lds_read<float4>((base ^ (ks << 6)) + row * ROW), b = lds_read<float4>((base ^ (ks << 6 | 16)) + row * ROW);
      f.v[0] = a.x; f.v[1] = a.y; f.v[2] = a.z; f.v[3] = a.w;
      f.v[4] = b.x; f.v[5] = b.y; f.v[6] = b.z; f.v[7] = b.w;
    }
#endif
    return f;
  }
  // feature 32 i + lane % 32 of the 16 rows from `row` (a multiple of 16) on, in the order of a result's registers: element e is row
  // 8 (e >> 2) + 4 (lane / 32) + (e & 3)
  __device__ static __forceinline__ Frag<T> col_frag(const char* lds, int row, int i) {
    Frag<T> f;
#if defined(__HIP_DEVICE_COMPILE__)
    const int lane = threadIdx.x & 63, h = lane >> 5;
    if constexpr (sizeof(T) == 2) {
      const int s = lane & 15, piece = 2 * ((lane >> 4) & 1) + ((s & 3) >> 1), k = 4 * h + (s >> 2);
      const uint32_t base = lds_address(lds) + k * ROW + ((piece ^ swz(k)) << 4) + 8 * (s & 1);
      shortx4_t v[2];
#pragma unroll
      for (int r = 0; r < 2; ++r)
        v[r] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) shortx4_t*)(uintptr_t)((base ^ (i << 6 | r << 5)) + (row + 8 * r) * ROW));
      struct { shortx4_t lo, hi; } both = {v[0], v[1]};
      f.v = __builtin_bit_cast(bf16x8_t, both);
    } else {
      const int d = lane & 31;
      const uint32_t base = lds_address(lds) + 4 * h * ROW + (((d >> 2) ^ (h << 3)) << 4) + 4 * (d & 3);
#pragma unroll
      for (int e = 0; e < 8; ++e) f.v[e] = lds_read<float>((base ^ (i << 7 | e << 4)) + (row + 8 * (e >> 2) + (e & 3)) * ROW);
    }
#endif
    return f;
  }
};

// everything that was copied and read is there, for all wavefronts of the block
__device__ __forceinline__ void tile_sync() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
#endif
}

// A result of the matrix cores is there 19 wait states after the instruction, and the compiler counts them on one of the ways that lead
// to a reader only (of a tile of 32 keys the last register was read too early behind a skipped branch).  So whatever reads results stands
// in one block with the products, or behind this.
__device__ __forceinline__ void results_settle() {
#if defined(__HIP_DEVICE_COMPILE__)
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
#endif
}

// a value and that of the other half of the wavefront, lane l ^ 32's
__device__ __forceinline__ float2 halves(float v) {
#if defined(__HIP_DEVICE_COMPILE__)
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return make_float2(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return make_float2(v, v);
#endif
}
__device__ __forceinline__ float half_max(float v) {
  const float2 h = halves(v);
  return fmaxf(h.x, h.y);
}
__device__ __forceinline__ float half_sum(float v) {
  const float2 h = halves(v);
  return h.x + h.y;
}

// the sum of eight of a result's registers
__device__ __forceinline__ float sum8(const floatx16_t& c, int half) {
  const int i = 8 * half;
  return ((c[i] + c[i + 1]) + (c[i + 2] + c[i + 3])) + ((c[i + 4] + c[i + 5]) + (c[i + 6] + c[i + 7]));
}
// the sum of a result's registers, pairs first
__device__ __forceinline__ float sum16(const floatx16_t& c) {
  float v[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = c[2 * i] + c[2 * i + 1];
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// four neighbouring elements of a result's column, as features of a row
template <typename T>
__device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
  if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
  else *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
}
// a result tile whose columns are tokens and whose rows are features 32 i .. + 31: times f into row p of `dim` features
template <typename T>
__device__ __forceinline__ void store_col(T* p, const floatx16_t& c, int i, int dim, float f) {
#pragma unroll
  for (int r = 0; r < 16; r += 4) {
    const int d = 32 * i + result_row(r);
    if (d < dim) store4(p + d, c[r] * f, c[r + 1] * f, c[r + 2] * f, c[r + 3] * f);
  }
}

// Tiles of BN keys that some of the positions p0 .. p1 see: those of the first `sinks` keys, then those of the window
struct KeyTiles {
  int sink, first, count;                             // tiles of the sinks that lie before tile `first`; tiles in all
  __device__ __forceinline__ KeyTiles(const AttnMask& m, int keys, int p0, int p1, int bn) {
    int lo = 0, hi = keys;
    if (m.window) {
      lo = p0 - m.window + 1;
      hi = p1 + m.window < hi ? p1 + m.window : hi;
      if (hi < m.sinks) hi = m.sinks < keys ? m.sinks : keys;
    }
    if (m.causal && p1 + 1 < hi) hi = p1 + 1;
    if (hi < 0) hi = 0;
    if (lo < 0) lo = 0;
    if (lo > hi) lo = hi;
    first = lo / bn;
    const int s = m.window && m.sinks > 0 ? (m.sinks - 1) / bn + 1 : 0;
    if (s >= first) {
      if (s > 0) first = 0;
      sink = 0;
    } else {
      sink = s;
    }
    count = (hi + bn - 1) / bn - first;
    if (count < 0) count = 0;
    count += sink;
  }
  __device__ __forceinline__ int tile(int t) const { return t < sink ? t : first + t - sink; }
};

struct AttnArgs {
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;
  Packed qs, ks;
  int heads, group, dim;                             // query heads, of them for one key head, features of a head
  AttnMask mask;
  float scale;
};
template <typename T>
constexpr int kKeyStage = sizeof(T) == 2 ? 64 : 32;    // keys of a stage of LDS
constexpr int kWaves = 4;                              // of a block, each with 32 rows of scores
// what a wavefront holds fits 256 registers: two a SIMD
template <typename T, int DP>
constexpr bool kTwoWaves = sizeof(T) == 2 || DP <= 64;

// Rows of a wavefront in a block of four, each with 32 queries of a head: hb (1, 2 or 4) of the heads that share keys, 128 / hb queries.
// Blocks that share keys are neighbours, late tiles (the long ones under a causal mask) come first.
struct HeadTile {
  int2 queries, keys;                                // rows of the sequence: first, count
  int kvh, head, shift, block_row, block_rows, row;  // row: the wavefront's first query
  __device__ __forceinline__ bool find(const AttnArgs& a, int hb, int tiles, int wave) {
    const int id = xcd_contiguous_index(blockIdx.x, gridDim.x);
    const int groups = a.group / hb, per_head = tiles * groups, at = id % per_head, bq = 32 * kWaves / hb;
    kvh = id / per_head;
    head = kvh * a.group + at % groups * hb + wave % hb;
    int seq, tile;
    if (!find_tile(a.qs, bq, tiles - 1 - at / groups, &seq, &tile)) return false;
    queries = a.qs.place(seq);
    keys = a.ks.place(seq);
    shift = keys.y - queries.y;
    block_row = tile * bq;
    block_rows = min(bq, queries.y - block_row);
    row = block_row + wave / hb * 32;
    return true;
  }
  __device__ __forceinline__ bool in(int lane) const { return row + (lane & 31) < queries.y; }
  __device__ __forceinline__ int64_t token(int lane) const { return (int64_t)queries.x + row + (lane & 31); }
  __device__ __forceinline__ int rows_left() const { return queries.y - row; }
};

// one copy of 16 bytes a lane (see dma16) from a base that the wavefront shares and an offset of the lane's own
__device__ __forceinline__ void dma16_at(const char* base, uint32_t offset, char* lds_dst) {
  const uint32_t m = (uint32_t)(uintptr_t)(lds_ptr_t)lds_dst;
  asm volatile("s_mov_b32 m0, %0" ::"s"(m) : "m0");
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(offset), "s"(base));
}

// Copies of ROWS rows of a matrix into a tile by the block.  Rows that all exist, less than 2^31 bytes apart in all: a scalar address and
// a lane's offset, which stay the same from tile to tile; features behind the last are the first ones again (the other operand is zero there,
// or what they add to is not stored).  Others choose between the row and zeros lane by lane.
template <typename T, int DP, int ROWS, int NW = kWaves>
struct RowCopies {
  using R = RowTile<T, DP>;
  static constexpr int N = ROWS / R::RPI / NW;
  static_assert(N * R::RPI * NW == ROWS, "whole copies");
  int64_t ld;                                        // bytes
  int pieces;
  bool plain;
  static constexpr bool SAME = NW * R::RPI % 16 == 0;           // the swizzle of a wavefront's copies: one offset serves all
  uint32_t at[SAME ? 1 : N];
  __device__ __forceinline__ RowCopies(int64_t ld_elements, int dim, int wave)
      : ld(ld_elements * (int)sizeof(T)), pieces(dim * (int)sizeof(T) / 16), plain(ld * ROWS < (INT64_C(1) << 31)) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < (SAME ? 1 : N); ++s) {
      const int row = (wave + NW * s) * R::RPI + lane / R::CH;
      const int piece = (lane % R::CH) ^ R::swz(row);
      at[s] = (uint32_t)(row * ld) + (piece < pieces ? piece << 4 : 0);
    }
  }
  // base: the tile's first row, of which `valid` exist; zeroed: with zeros behind the last feature
  __device__ __forceinline__ void issue(const char* base, int valid, char* lds, int wave, bool zeroed = false) const {
    if (plain && valid >= ROWS && !zeroed) {
#pragma unroll
      for (int s = 0; s < N; ++s) dma16_at(SAME ? base + s * NW * R::RPI * ld : base, at[SAME ? 0 : s], lds + (wave + NW * s) * 1024);
    } else {
#pragma unroll
      for (int s = 0; s < N; ++s) R::copy(base, ld, valid, pieces, lds, wave + NW * s);
    }
  }
};
// of a stage's keys and values
template <typename T, int DP, int BN>
struct KeyCopies {
  using R = RowTile<T, DP>;
  const char *k, *v;
  RowCopies<T, DP, BN> ck, cv;
  int keys;
  __device__ __forceinline__ KeyCopies(const AttnArgs& a, int2 place, int kvh, int wave)
      : k((const char*)((const T*)a.k + (int64_t)place.x * a.ldk + kvh * a.dim)), v((const char*)((const T*)a.v + (int64_t)place.x * a.ldv + kvh * a.dim)),
        ck(a.ldk, a.dim, wave), cv(a.ldv, a.dim, wave), keys(place.y) {}
  __device__ __forceinline__ void issue_keys(int tile, char* buf, int wave) const { ck.issue(k + tile * BN * ck.ld, keys - tile * BN, buf, wave); }
  __device__ __forceinline__ void issue_values(int tile, char* buf, int wave) const { cv.issue(v + tile * BN * cv.ld, keys - tile * BN, buf, wave); }
  __device__ __forceinline__ void issue(int tile, char* buf, int wave) const {
    issue_keys(tile, buf, wave);
    issue_values(tile, buf + BN * R::ROW, wave);
  }
};

// A wavefront's 32 tokens (columns) of DP features times f, `rows` of them, into rows of memory.  bf16: through its own 8 (4) KB of LDS, so that
// 16 bytes of a row leave at once and neighbouring lanes write neighbouring pieces; fp32: four features are 16 bytes as they are.
template <typename T, int DP>
__device__ __forceinline__ void store_rows(T* to, int64_t ld, int rows, int dim, const floatx16_t (&acc)[DP / 32], float f, char* lds) {
  const int lane = threadIdx.x & 63;
  if constexpr (sizeof(T) == 4) {
    if ((lane & 31) < rows) {
#pragma unroll
      for (int i = 0; i < DP / 32; ++i) store_col(to + (lane & 31) * ld, acc[i], i, dim, f);
    }
  } else {
    constexpr int CH = RowTile<T, DP>::PITCH / 8;
    const int r = lane & 31;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int x = 0; x < 16; x += 4) {
        const int d = 32 * i + result_row(x);          // four features: half a piece
        store4((T*)(lds + r * CH * 16 + (((d >> 3) ^ (r & (CH - 1))) << 4) + 2 * (d & 7)), acc[i][x] * f, acc[i][x + 1] * f, acc[i][x + 2] * f, acc[i][x + 3] * f);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int s = 0; s < 32 * CH / 64; ++s) {
      const int row = s * (64 / CH) + lane / CH, piece = lane % CH;
      const uint4 v = *(const uint4*)(lds + row * CH * 16 + ((piece ^ (row & (CH - 1))) << 4));
      if (row < rows && piece * 8 < dim) *(uint4*)(to + row * ld + piece * 8) = v;
    }
  }
}

// ---- host side
constexpr int64_t kAttnMostBlocks = (1 << 24) - 1;    // of 256 lanes: a grid has fewer than 2^32
// rows of heads: at least `cols` wide, in whole 16 bytes from a 16-byte aligned address
inline int attn_rows(const void* p, int64_t ld, int64_t cols, int dtype) {
  if (ld < cols || ld > (INT64_C(1) << 24)) return EFQAT_ERR_BAD_SHAPE;
  if (!p) return EFQAT_ERR_NULL_PTR;
  if (!aligned16(p) || ld % (dtype == EFQAT_F32 ? 4 : 8)) return EFQAT_ERR_ALIGNMENT;
  return EFQAT_OK;
}
// results that lie where operands do, which blocks and kernels behind the one that writes them still read
inline int attn_apart(std::initializer_list<const void*> results, std::initializer_list<const void*> operands) {
  for (const void* r : results)
    for (const void* o : operands)
      if (r == o) return EFQAT_ERR_BAD_LAYOUT;
  return EFQAT_OK;
}
inline int attn_args(AttnArgs* a, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int64_t Tq,
                     int64_t Tk, int64_t n_seq, const int32_t* q_start, const int32_t* k_start, int64_t heads, int64_t kv_heads, int64_t dim,
                     float scale, int causal, int64_t window, int64_t sinks) {
  if (Tq <= 0 || Tk <= 0 || Tq > kAttnMostRows || Tk > kAttnMostRows || n_seq <= 0 || n_seq > (1 << 24) || heads <= 0 || kv_heads <= 0 ||
      heads > 65535 || heads % kv_heads || dim <= 0 || dim > 128 || dim % 8 || window < 0 || sinks < 0)
    return EFQAT_ERR_BAD_SHAPE;
  if (!(scale > 0.0f) || !(scale < INFINITY)) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (causal != 0 && causal != 1) return EFQAT_ERR_BAD_LAYOUT;
  if (!q_start != !k_start) return EFQAT_ERR_NULL_PTR;                    // both packed by offsets, or both evenly
  if (!q_start && (Tq % n_seq || Tk % n_seq)) return EFQAT_ERR_BAD_SHAPE;
  EFQAT_TRY(attn_rows(q, ldq, heads * dim, dtype));
  EFQAT_TRY(attn_rows(k, ldk, kv_heads * dim, dtype));
  EFQAT_TRY(attn_rows(v, ldv, kv_heads * dim, dtype));
  if (!aligned4(q_start) || !aligned4(k_start)) return EFQAT_ERR_ALIGNMENT;
  const int64_t far = kAttnMostRows;
  *a = {q, k, v, ldq, ldk, ldv, {q_start, (int)Tq, (int)n_seq}, {k_start, (int)Tk, (int)n_seq}, (int)heads, (int)(heads / kv_heads), (int)dim,
        {causal, window >= far ? 0 : (int)window, sinks >= far ? (int)far : (int)sinks}, scale};
  return EFQAT_OK;
}

// Blocks of the kernels that walk keys
struct HeadPlan {
  int hb, tiles;
  int64_t blocks;
};
inline HeadPlan head_plan(const AttnArgs& a, int64_t kv_heads) {
  int hb = 1;
  while (hb < kWaves && a.group % (2 * hb) == 0) hb *= 2;
  const int64_t tiles = a.qs.most_tiles(32 * kWaves / hb);
  return {hb, (int)tiles, tiles * (a.group / hb) * kv_heads};
}

}  // namespace efqat
