// The three products of the loss over a vocabulary, on bf16 operands with fp32 sums:
//
//   out[n][m] = sum_k A[m][k] B[n][k]
//
//   logits (XG_LSE, XG_GRAD, XG_GRAD3 for G in three parts, XG_PART)  A = class weights W [m = class][k = feature], B = features H [n = token][k]
//   dH     (XG_DH)            A = W read as [k = class][m = feature], B = G [n = token][k = class]
//   dW     (XG_DW)            A = H read as [k = token][m = feature], B = G read as [k = token][n = class]
//
// An operand whose contraction index is its row (TR) is copied into LDS as it lies and transposed by the LDS reads
// (ds_read_b64_tr_b16), so that no transposed copy of W, H or G exists.  With classes along m and tokens along n the accumulators
// of a lane are classes of one token: the softmax statistics of a token are sums over registers and one exchange between the two
// halves of a wavefront, instead of a reduction over 32 lanes for every row.
//
// Square tiles: 256 by eight wavefronts of 128 x 64 (the accumulators are half of a lane's registers, two wavefronts a SIMD),
// 128 by four of 64 x 64.  K stages of 64 in two LDS buffers; a stage's copies go out in the last sub-step of the stage before the
// previous one's end and in the first of the previous, so that they have two sub-steps to land; fragment reads run a sub-step ahead
// of the matrix instructions.  The order is pinned, one group per matrix instruction.  64 by four wavefronts that each walk K stages of
// their own.
//
// Bound by the matrix cores where the tiles are large: 8028 tokens of width 4096 against 32000 classes (2.1 T operations a product), the
// logits with their sums 1.58 ms (1.33 POP/s; a library product of 8192^3 reaches 1.38), the logits and G 1.67 ms (1.26), both products of
// G 3.23 ms (1.30).  A 256-tile of logits costs 1.6 us a K stage and 5.5 us besides (128 exponentials a lane in the epilogue, the first
// loads): 12 stages, as in a width of 768, reach 0.87 POP/s.  The epilogues are written so that no accumulator changes under a branch (copies
// of all of them) and their addresses are not kept through the products: 217 registers, no spills; with both, G's had 256 and spilled, and
// 1843 tokens of width 768 against 30522 classes took 313 us backward instead of 291.  A round of four stages of a 64-tile takes 0.67 us, which the copies into LDS
// (64 KB at 64 bytes a clock: 0.43 us) are most of.  LDS bank conflicts: none in the products and the softmax sums (counted); in the epilogues
// that lay out G and bf16 results, 1 to 3 % of all LDS cycles at a width of 4096, 3 to 13 % at 768 and below.
//
// fp32 operands are three bf16 parts each (x = x0 + x1 + x2 with 24 bits), side by side in a row; the product of two is the six
// largest of the nine products of parts, smallest first: `segments` walks them, each a contraction of its own over the same rows.
// What is left out is below 2^-24 of the product of the magnitudes.
#pragma once
#include "rows.hpp"

#include <type_traits>

#include "gemm_epilogue.hpp"
#include "lds_copy.hpp"

namespace efqat {

enum XentMode { XG_LSE = 0, XG_GRAD = 1, XG_DH = 2, XG_DW = 3, XG_PART = 4, XG_GRAD3 = 5 };

// The classes are taken in pieces, whose size follows from the number of tokens that have a class: a piece's G has about `elems`
// elements (of all its parts), and its classes, where they are laid out anew, are `cap` at most.  The host knows the number of tokens
// only as a limit and launches the pieces that the limit needs; the last of them may find nothing left.
struct XentPieces {
  int V, cap;
  uint32_t elems;                 // 0: no limit but cap
  int parts;
  __host__ __device__ int size(int tokens) const {
    const uint32_t slots = tokens < 1 ? 256u : ((uint32_t)tokens + 255u) / 256u * 256u;
    uint32_t most = (uint32_t)cap;
    if (elems) {
      const uint32_t fit = elems / (slots * (uint32_t)parts) / 256u * 256u;       // slots * parts < 2^32: check_xent
      most = fit < 1024u ? 1024u : fit;
      most = most < (uint32_t)cap ? most : (uint32_t)cap;
    }
    const uint32_t n = ((uint32_t)V + most - 1u) / most, even = ((uint32_t)V + n - 1u) / n;
    return (int)((even + 255u) / 256u * 256u);
  }
};

struct XentGemmArgs {
  const bf16_t *W, *H;            // operands in whole stages: [class][parts][Dp] (W: of all classes, or of the piece alone), [slot][parts][Dp]
  bf16_t* G;                      // [slot][parts][piece]
  int w_piece;                    // 1: W holds the piece alone, zeros behind its last class
  int64_t ldw, Dp;                // elements between the rows of W; features in whole stages
  int64_t D;
  int segments;                   // 1, or 6 products of parts
  XentPieces pieces;
  int piece;                      // number of the piece
  const int32_t* n_valid;
  int split_blocks;               // XG_PART and products of G: K is cut so that about that many blocks work (xent_split)
  // logits, per token slot
  const int32_t* target;
  float2* part;                   // XG_LSE: [tile of classes][slots] (largest logit, sum of exp(logit - largest))
  float* target_logit;            // XG_LSE
  int64_t slots;
  const float *lse, *scale;       // XG_GRAD, by slot; scale NULL: ones
  // XG_PART and products of G: fp32 partial results [slice][n][M], and the output; the result is multiplied by *factor (NULL: 1), and divided by the
  // number of tokens (mean)
  const float* factor;
  int mean;
  float* acc;
  void* out;
  int out_dtype;
  int64_t ldo;
  const int32_t* rows;            // XG_DH: rows of the output, by slot
};

// Slices of K of a product of so many tiles: about `blocks` blocks, none with fewer than 12 stages.  Shorter ones cost more at the
// join than they save, longer ones leave CUs without work: at least 6 / 12 / 24 stages, backward of 256 fp32 tokens of width 256 against
// 1000 classes 37.6 / 31.8 / 30.7 us, of 128 of 1920 against 786 71.2 / 71.2 / 72.9, of 65 bf16 of 768 against 30522 73.0 / 66.5 / 69.7.
__host__ __device__ inline int xent_split(int64_t tiles, int stages, int segments, int blocks) {
  const int by_blocks = tiles > blocks || tiles < 1 ? 1 : blocks / (int)tiles;
  const int by_stages = (int)((int64_t)stages * segments / 12);
  const int s = by_blocks < by_stages ? by_blocks : by_stages;
  return s < 1 ? 1 : s;
}

// Sizes of a product, from the number of tokens
struct XentShape {
  int64_t class0;
  int classes, piece;             // of this piece (0: nothing left), of a whole one
  int M, N, K, nks;               // nks: stages of a segment
  int split_stages, split_n;
  __device__ __forceinline__ int split_tiles(int bt) const { return ((M + bt - 1) / bt) * ((split_n + bt - 1) / bt); }
  __device__ __forceinline__ XentShape(const XentGemmArgs& g, XentMode mode, int valid) {
    piece = __builtin_amdgcn_readfirstlane(g.pieces.size(valid));
    class0 = (int64_t)piece * g.piece;
    const int64_t left = g.pieces.V - class0;
    classes = (int)(left < 0 ? 0 : left < piece ? left : piece);
    M = mode == XG_DH || mode == XG_DW ? (int)g.D : classes;
    N = mode == XG_DW ? classes : valid;
    K = mode == XG_DW ? valid : mode == XG_DH ? classes : (int)g.Dp;
    nks = (K + 63) / 64;
    // slices by a whole piece: dH adds those of the last, shorter one to the same partial results
    const int whole = piece < g.pieces.V ? piece : g.pieces.V;
    split_stages = mode == XG_DH ? (whole + 63) / 64 : nks;
    split_n = mode == XG_DW ? whole : N;
  }
};

// One wave-wide global -> LDS copy (see dma16) from a uniform base and 32-bit offsets
__device__ __forceinline__ void dma16_at(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %0" ::"s"(lds) : "m0");
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base));
}

typedef int intx4_xg_t __attribute__((ext_vector_type(4)));

// One operand of a tile: BW rows (or columns, TR) of the tile, WW of them a wavefront's
template <int BW, int WW, int NW, bool TR>
struct XentOperand {
  static constexpr int T = WW / 32;                   // fragments of a wavefront and sub-step
  static constexpr int G = BW / 8 / NW;               // 1-KiB copies of a wavefront and stage
  static constexpr int RB = 2 * BW;                   // TR: bytes of an LDS row
  static constexpr int CPR = RB / 16, RPC = 1024 / RB; // TR: chunks of a row, rows of a copy
  static constexpr int READS = TR ? 2 * T : T;
  static constexpr int ADDR = TR ? T : 4;
  uint32_t voff[G];
  int addr[ADDR];
  struct Frag { intx4_xg_t v; };

  // physical 16-byte chunk of an LDS row: reads of half a wavefront touch all banks once
  __device__ static __forceinline__ int swz(int c, int k) { return c ^ (4 * (BW == 64 ? (k >> 1) & 1 : k & 3)); }

  // limit: rows (columns, TR) of the tile that exist; the others repeat one that does, their results are dropped
  __device__ __forceinline__ void setup(int64_t ld, int limit, int wave, int wpos, int lane, int lds0) {
    const uint32_t ld2 = (uint32_t)(ld * 2);
#pragma unroll
    for (int j = 0; j < G; ++j) {
      const int u = wave + NW * j;
      if constexpr (TR) {
        const int k = u * RPC + lane / CPR;
        int col = swz(lane % CPR, k) * 8;
        col = col < limit ? col : 0;
        voff[j] = (uint32_t)k * ld2 + (uint32_t)col * 2;
      } else {
        const int r = u * 8 + (lane >> 3);
        const int c = (lane & 7) ^ ((r >> 1) & 7);
        voff[j] = (uint32_t)(r < limit ? r : limit - 1) * ld2 + (uint32_t)c * 16;
      }
    }
    if constexpr (TR) {
      const int s = lane & 15, q = lane >> 4, mb = 16 * (q & 1), h = q >> 1, k = 8 * h + (s >> 2);
#pragma unroll
      for (int i = 0; i < T; ++i) {
        const int c = (wpos * WW + 32 * i + mb + 4 * (s & 3)) >> 3;
        addr[i] = lds0 + k * RB + (swz(c, k) << 4) + 8 * (s & 1);
      }
    } else {
      const int fr = lane & 31, fh = lane >> 5;
#pragma unroll
      for (int sub = 0; sub < 4; ++sub)
        addr[sub] = lds0 + (wpos * WW + fr) * 128 + (((2 * sub + fh) ^ ((fr >> 1) & 7)) << 4);
    }
  }
  // copy j of a stage; last: of a TR operand, rows k >= left do not exist, the last one is repeated (the other operand's are zero); of
  // another, columns >= left (whole chunks) do not, they are zeros
  __device__ __forceinline__ void copy(const char* base, uint32_t lds, int wave, int j) const {
    dma16_at(base, voff[j], lds + (wave + NW * j) * 1024);
  }
  __device__ __forceinline__ void copy_last(const char* base, uint32_t lds, int wave, int lane, int j, int64_t ld, int left) const {
    uint32_t off = voff[j];
    if constexpr (TR) {
      const int k = (wave + NW * j) * RPC + lane / CPR;
      if (k >= left) off -= (uint32_t)(k - left + 1) * (uint32_t)(ld * 2);
      dma16_at(base, off, lds + (wave + NW * j) * 1024);
    } else {
      const int r = (wave + NW * j) * 8 + (lane >> 3), c = (lane & 7) ^ ((r >> 1) & 7);
      const char* from = c * 8 < left ? base + off : zero_page();
      asm volatile("s_mov_b32 m0, %0" ::"s"(lds + (wave + NW * j) * 1024) : "m0");
      asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from));
    }
  }
  // read number r of sub-step sub
  __device__ __forceinline__ void read(const char* smem, int sub, int r, Frag (&f)[T]) const {
    if constexpr (TR) {
      const int i = r >> 1, hh = r & 1;
      const shortx4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (__attribute__((address_space(3))) shortx4_t*)(smem + addr[i] + sub * 16 * RB + hh * 4 * RB));
      const intx2_t w = __builtin_bit_cast(intx2_t, v);
      f[i].v[2 * hh] = w[0];
      f[i].v[2 * hh + 1] = w[1];
    } else {
      f[r].v = *reinterpret_cast<const intx4_xg_t*>(smem + addr[sub] + r * 4096);
    }
  }
  __device__ __forceinline__ void other_buffer(int stage_bytes) {
#pragma unroll
    for (int i = 0; i < ADDR; ++i) addr[i] ^= stage_bytes;
  }
};

template <int BT>
struct XentCfg {
  static constexpr int NW = BT == 256 ? 8 : 4, WGM = 2, WGN = NW / 2;       // wavefronts of a tile
  static constexpr int THREADS = NW * 64;
  static constexpr int CHIP = BT == 128 ? 512 : 256;  // blocks that the chip holds at once
  static constexpr int WM = BT / WGM, WN = BT / WGN, TM = WM / 32, TN = WN / 32;
  static constexpr int STAGE = BT * 256;              // bytes of both operands' stage, a power of two
  static constexpr bool OWN = BT == 64;               // every wavefront works on K stages of its own, of the whole tile
  static constexpr int RINGS = OWN ? NW : 1;          // rings of two LDS stages
  static constexpr int OUT_PITCH = WM * 2 + 16;       // bytes of a row of a wavefront's bf16 results in LDS
  static constexpr int LDS = RINGS * 2 * STAGE > NW * WN * OUT_PITCH ? RINGS * 2 * STAGE : NW * WN * OUT_PITCH;
};

// bf16 parts of x: x0 + x1 + x2 = x up to 2^-24.  A NaN is its first part.  What bf16 has no finite value for, infinities among it,
// is the largest one it has: an infinite first part times another operand's zero part would be a NaN in every product.
__device__ __forceinline__ void split3(float x, float (&p)[3]) {
  constexpr float kMost = 0x1.FEp127f;
  x = fabsf(x) > kMost ? copysignf(kMost, x) : x;
  p[0] = __uint_as_float(pack_bf16x2(x, x) << 16);
  const float r1 = p[0] == p[0] ? x - p[0] : 0.0f;
  p[1] = __uint_as_float(pack_bf16x2(r1, r1) << 16);
  p[2] = r1 - p[1];
}

// Tiles of a product (times its slices of K)
struct XentTiles {
  int m, n, slices;
  __device__ __forceinline__ XentTiles(const XentGemmArgs& g, const XentShape& z, XentMode mode, int bt) {
    m = (z.M + bt - 1) / bt;
    n = (z.N + bt - 1) / bt;
    const bool cut = mode == XG_DH || mode == XG_DW || mode == XG_PART;
    slices = cut ? __builtin_amdgcn_readfirstlane(xent_split(z.split_tiles(bt), z.split_stages, g.segments, g.split_blocks)) : 1;
  }
  __device__ __forceinline__ int total() const { return m * n * slices; }
};

// one tile (and slice) of a product: number `bid` of them in the order of the launch
template <int BT, XentMode MODE>
__device__ __forceinline__ void xent_gemm_block(const XentGemmArgs& g, const XentShape& z, const XentTiles& tiles_of, int valid, int bid, char* smem) {
#if defined(__HIP_DEVICE_COMPILE__)
  using C = XentCfg<BT>;
  constexpr bool GRAD = MODE == XG_GRAD || MODE == XG_GRAD3, LOGITS = MODE == XG_LSE || GRAD || MODE == XG_PART, SOFT = MODE == XG_LSE || GRAD;
  constexpr bool ATR = !LOGITS, BTR = MODE == XG_DW;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / C::WGN, wn = wave % C::WGN;

  const int M = z.M, N = z.N, nks = z.nks;
  const int tiles_m = tiles_of.m, tiles_n = tiles_of.n, nslice = tiles_of.slices, tiles = tiles_m * tiles_n, total = tiles * nslice;
  // neighbours run on one XCD, in groups of 4 rows of tiles
  const int logical = xcd_contiguous_index(bid, total);
  const int slice = logical / tiles, pid = logical - slice * tiles;
  constexpr int GM = 4;
  const int per_group = GM * tiles_n, group = pid / per_group, first_m = group * GM;
  const int gsize = tiles_m - first_m < GM ? tiles_m - first_m : GM;
  const int tm = __builtin_amdgcn_readfirstlane(first_m + (pid % per_group) % gsize);
  const int tn = __builtin_amdgcn_readfirstlane((pid % per_group) / gsize);
  const int m0 = tm * BT, n0 = tn * BT;
  const int k_first = __builtin_amdgcn_readfirstlane((int)((int64_t)nks * slice / nslice));
  const int k_end = __builtin_amdgcn_readfirstlane((int)((int64_t)nks * (slice + 1) / nslice));
  const int per_seg = k_end - k_first, nstage = per_seg * g.segments;

  const int parts = g.segments == 6 ? 3 : 1;
  const int64_t ldh = parts * g.Dp, ldg = (int64_t)parts * z.piece;
  const bf16_t* W = g.W + (g.w_piece ? 0 : z.class0 * g.ldw);
  const bf16_t* opA = MODE == XG_DW ? g.H : W;
  const bf16_t* opB = LOGITS ? g.H : g.G;
  const int64_t lda = MODE == XG_DW ? ldh : g.ldw, ldb = LOGITS ? ldh : ldg;
  const int64_t a_part = g.Dp, b_part = LOGITS ? g.Dp : z.piece;
  // classes as they lie end inside the last stage: rows in dH, columns in the logits
  const int a_end = g.w_piece || MODE == XG_DW ? 0 : MODE == XG_DH ? z.K : (int)g.D;

  // what the epilogue needs of the tokens: on its way while the product runs
  const int n_lane = n0 + wn * C::WN + (lane & 31);
  int tok_class[SOFT ? C::TN : 1];
  float tok_lse[GRAD ? C::TN : 1], tok_scale[GRAD ? C::TN : 1];
  if constexpr (SOFT) {
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      const int n = n_lane + 32 * j;
      tok_class[j] = n < N ? g.target[n] : -1;
      if constexpr (GRAD) {
        tok_lse[j] = n < N ? g.lse[n] : 0.0f;
        tok_scale[j] = n < N && g.scale ? g.scale[n] : 1.0f;
      }
    }
  }

  XentOperand<BT, C::OWN ? BT : C::WM, C::OWN ? 1 : C::NW, ATR> A;
  XentOperand<BT, C::OWN ? BT : C::WN, C::OWN ? 1 : C::NW, BTR> B;
  const int copier = C::OWN ? 0 : wave;               // among the wavefronts that copy a stage together
  A.setup(lda, ATR ? (int)g.D - m0 : M - m0, copier, C::OWN ? 0 : wm, lane, 0);
  B.setup(ldb, BTR ? z.piece - n0 : N - n0, copier, C::OWN ? 0 : wn, lane, BT * 128);
  const int64_t a_step = ATR ? lda * 128 : 128, b_step = BTR ? ldb * 128 : 128;
  const char* a_base = (const char*)opA + (ATR ? (int64_t)m0 * 2 : (int64_t)m0 * lda * 2) + k_first * a_step;
  const char* b_base = (const char*)opB + (BTR ? (int64_t)n0 * 2 : (int64_t)n0 * ldb * 2) + k_first * b_step;
  // the copy stream: stage, its place in its segment, its sources
  int c_seg = 0, c_kt = 0;
  auto seg_a = [&](int s) { return (int)((0x001102u >> (4 * (g.segments == 6 && s < 5 ? s : 5))) & 15u); };
  auto seg_b = [&](int s) { return (int)((0x010120u >> (4 * (g.segments == 6 && s < 5 ? s : 5))) & 15u); };
  const char* a_src = a_base + (int64_t)seg_a(0) * a_part * 2;
  const char* b_src = b_base + (int64_t)seg_b(0) * b_part * 2;
  auto next_stage = [&]() {
    if (++c_kt == per_seg) {
      c_kt = 0;
      ++c_seg;
      a_src = a_base + (int64_t)seg_a(c_seg) * a_part * 2;
      b_src = b_base + (int64_t)seg_b(c_seg) * b_part * 2;
    } else {
      a_src += a_step;
      b_src += b_step;
    }
  };
  constexpr int AG = decltype(A)::G, BG = decltype(B)::G, LPS = AG + BG, H0 = (LPS + 1) / 2;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
  auto issue = [&](auto lastc, int buf, int t0, int t1) {
    const uint32_t l = lds0 + buf * C::STAGE;
#pragma unroll
    for (int t = t0; t < t1; ++t) {
      if (t < AG) {
        if constexpr (decltype(lastc)::value) A.copy_last(a_src, l, copier, lane, t, lda, a_end - (k_end - 1) * 64);
        else A.copy(a_src, l, copier, t);
      } else {
        B.copy(b_src, l + BT * 128, copier, t - AG);
      }
    }
  };
  using Last = std::integral_constant<bool, true>;
  using Whole = std::integral_constant<bool, false>;
  // the last stage is copied apart if they do
  const int nfull = a_end && k_end == nks && (a_end & 63) ? nstage - 1 : nstage;

  floatx16_t acc[C::TM][C::TN];
#pragma unroll
  for (int i = 0; i < C::TM; ++i)
#pragma unroll
    for (int j = 0; j < C::TN; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

  constexpr int TM = decltype(A)::T, TN = decltype(B)::T;             // fragments of a wavefront in the product
  typename decltype(A)::Frag af[2][TM];
  typename decltype(B)::Frag bf[2][TN];
  constexpr int RA = decltype(A)::READS, RBR = decltype(B)::READS, NRD = RA + RBR, MF = TM * TN;
  auto read_one = [&](int sub, int rb, int r) {
    if (r < RBR) B.read(smem, sub, r, bf[rb]);
    else A.read(smem, sub, r - RBR, af[rb]);
  };
  auto read_all = [&](int sub, int rb) {
#pragma unroll
    for (int r = 0; r < NRD; ++r) read_one(sub, rb, r);
  };
  auto mfma_into = [&](floatx16_t& d, const auto& a, const auto& b) {
    d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a.v), __builtin_bit_cast(bf16x8_t, b.v), d, 0, 0, 0);
  };
  auto mfma_one = [&](int rb, int i, int j) { mfma_into(acc[i][j], af[rb][i], bf[rb][j]); };
  auto mfma_all = [&](int rb) {
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
      for (int j = 0; j < C::TN; ++j) mfma_one(rb, i, j);
  };
  // the copies of the next stage have landed, every wavefront has read all of this one's
  auto stage_sync = [&]() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    A.other_buffer(C::STAGE);
    B.other_buffer(C::STAGE);
  };
  // matrix instructions of fragment set rb; the reads of sub-step sub_next into the other set; copies t0 .. t1 - 1 into buf
  constexpr int RG = (2 * MF + 2) / 3;
  auto substep = [&](int sub_next, int rb, int buf, int t0, int t1) {
#pragma unroll
    for (int q = 0; q < MF; ++q) {
      mfma_one(rb, q / C::TN, q % C::TN);
      if (q < RG) {
#pragma unroll
        for (int r = (q * NRD) / RG; r < ((q + 1) * NRD) / RG; ++r) read_one(sub_next, rb ^ 1, r);
      }
      issue(Whole{}, buf, t0 + (t1 - t0) * q / MF, t0 + (t1 - t0) * (q + 1) / MF);
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  if constexpr (C::OWN) {
    // Few tiles: what counts is how long one takes.  Every wavefront walks K stages of its own, with all 64 x 64 results: a stage is read
    // from LDS once (wavefronts of 32 x 32 read it twice), and nobody waits for anybody at a barrier.  The copies of a stage are under way
    // while the one before is worked on.  128 fp32 tokens of width 1920 against 786 classes, forward: 49 us; two groups of four wavefronts
    // of 32 x 32 that take every other stage in rings of four: 62 us.
    const int mine = (nstage - wave + C::NW - 1) / C::NW, ring = wave * 2;           // stages of this wavefront
    floatx16_t own[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
      for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) own[i][j][r] = 0.0f;
    for (int k = 0; k < wave && k < nstage; ++k) next_stage();
    auto issue_stage = [&](int r) {
      if (r * C::NW + wave < nfull) issue(Whole{}, ring + (r & 1), 0, LPS);
      else issue(Last{}, ring + (r & 1), 0, LPS);
#pragma unroll
      for (int k = 0; k < C::NW; ++k) next_stage();
    };
    if (mine > 0) issue_stage(0);
    if (mine > 1) issue_stage(1);
    for (int r = 0; r < mine; ++r) {
      if (r + 1 < mine) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LPS) : "memory");
      else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
      const char* at = smem + (ring + (r & 1)) * C::STAGE;
      typename decltype(A)::Frag a4[4][TM];
      typename decltype(B)::Frag b4[4][TN];
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
#pragma unroll
        for (int q = 0; q < RBR; ++q) B.read(at, sub, q, b4[sub]);
#pragma unroll
        for (int q = 0; q < RA; ++q) A.read(at, sub, q, a4[sub]);
      }
#pragma unroll
      for (int sub = 0; sub < 4; ++sub) {
        if (sub == 3) {                               // everything has been read: the stage after the next takes the place
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_sched_barrier(0);
          if (r + 2 < mine) issue_stage(r + 2);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
          for (int j = 0; j < TN; ++j) mfma_into(own[i][j], a4[sub][i], b4[sub][j]);
      }
    }
    // each wavefront adds up 32 x 32 of the results, in the order of the wavefronts
    __syncthreads();
    float4* sum = reinterpret_cast<float4*>(smem);    // [wavefront][32 x 32][4][lane]
    if (mine > 0) {
#pragma unroll
      for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
          for (int q = 0; q < 4; ++q)
            sum[((wave * C::NW + i * C::WGN + j) * 4 + q) * 64 + lane] =
                make_float4(own[i][j][4 * q], own[i][j][4 * q + 1], own[i][j][4 * q + 2], own[i][j][4 * q + 3]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < C::NW; ++k) {
      if (k >= nstage) break;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const float4 v = sum[((k * C::NW + wave) * 4 + q) * 64 + lane];
        acc[0][0][4 * q] += v.x;
        acc[0][0][4 * q + 1] += v.y;
        acc[0][0][4 * q + 2] += v.z;
        acc[0][0][4 * q + 3] += v.w;
      }
    }
  } else
  // On entry to stage s the first H0 copies of stage s + 1 are under way if and only if s + 1 < nfull.
  if (nstage > 0) {
    if (nfull > 0) issue(Whole{}, 0, 0, LPS);
    else issue(Last{}, 0, 0, LPS);
    next_stage();
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (1 < nfull) issue(Whole{}, 1, 0, H0);
    read_all(0, 0);
    int s = 0, buf = 0;
    for (; s + 2 < nfull; ++s, buf ^= 1) {
      __builtin_amdgcn_sched_barrier(0);
      substep(1, 0, buf ^ 1, H0, LPS);
      next_stage();
      substep(2, 1, 0, 0, 0);
      substep(3, 0, 0, 0, 0);
      stage_sync();
      substep(0, 1, buf, 0, H0);
    }
    for (; s < nstage; ++s, buf ^= 1) {
      if (s + 1 < nfull) {
        issue(Whole{}, buf ^ 1, H0, LPS);
        next_stage();
      } else if (s + 1 < nstage) {
        issue(Last{}, buf ^ 1, 0, LPS);
        next_stage();
      }
      __builtin_amdgcn_sched_barrier(0);
      read_all(1, 1);
      mfma_all(0);
      __builtin_amdgcn_sched_barrier(0);
      read_all(2, 0);
      mfma_all(1);
      __builtin_amdgcn_sched_barrier(0);
      read_all(3, 1);
      mfma_all(0);
      stage_sync();
      if (s + 1 < nstage) read_all(0, 0);
      if (s + 2 < nfull) issue(Whole{}, buf, 0, H0);
      mfma_all(1);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  __syncthreads();

  // ---- accumulators: column n = lane & 31, rows m = 8 (r / 4) + 4 (lane / 32) + r % 4 of their 32 x 32
  int late = lane;                                    // not known to be the same for every tile: addresses that follow from it are made
  asm volatile("" : "+v"(late));                      // here, not kept in registers through the products
  const int fr = late & 31, fh = late >> 5;
  const int mw = m0 + wm * C::WM + 4 * fh, nw = n0 + wn * C::WN + fr;
  auto m_of = [&](int i, int r) { return mw + 32 * i + 8 * (r >> 2) + (r & 3); };

  if constexpr (MODE == XG_LSE) {
    // largest logit and sum of exponentials of the tile's classes, for every token; the tile's wavefronts join theirs in LDS
    float2* red = reinterpret_cast<float2*>(smem);    // [WGM][BT]
    if (m0 + BT > M) {                                // the last class is repeated
#pragma unroll
      for (int j = 0; j < C::TN; ++j)
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = m_of(i, r) < M ? acc[i][j][r] : -INFINITY;
    }
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
      const int n = nw + 32 * j;
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) top = fmaxf(top, acc[i][j][r]);
      top = fmaxf(top, __shfl_xor(top, 32));
      // a token whose logits are all -inf has sum 0; a NaN makes the sum NaN
      const float base = top == -INFINITY ? 0.0f : top;
      float sum = 0.0f;
#pragma unroll
      for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f((acc[i][j][r] - base) * 1.4426950408889634f);
      sum += __shfl_xor(sum, 32);
      if (fh == 0) red[wm * BT + wn * C::WN + 32 * j + fr] = make_float2(top, sum);
      const int rel = n < N ? tok_class[j] - (int)z.class0 - m0 - wm * C::WM : -1;   // row of the wavefront's tile that is the class
      if (__any(rel >= 0 && rel < C::WM)) {
        const int mine = rel - 4 * fh;
        float at_class = 0.0f;
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) at_class = mine == 32 * i + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : at_class;
        if (mine >= 0 && mine < C::WM && !(mine & 4)) g.target_logit[n] = at_class;
      }
    }
    __syncthreads();
    if (tid < BT && n0 + tid < N) {
      float2 a = red[tid];
      const float2 b = red[BT + tid];
      const float top = fmaxf(a.x, b.x), base = top == -INFINITY ? 0.0f : top;
      a.y = a.y * __builtin_amdgcn_exp2f((a.x - base) * 1.4426950408889634f) + b.y * __builtin_amdgcn_exp2f((b.x - base) * 1.4426950408889634f);
      a.x = top;
      g.part[(z.class0 / BT + tm) * g.slots + n0 + tid] = a;
    }
  } else {
    // a wavefront's results as rows of WM values in LDS, from where they leave 16 bytes a lane
    char* tile = smem + wave * (C::WN * C::OUT_PITCH);
    constexpr int CPR = C::WM * 2 / 16, RPI = 64 / CPR;            // chunks of a row, rows of an access
    auto put = [&](int i, int j, int q, float a, float b, float c, float d) {
      *reinterpret_cast<uint2*>(tile + (32 * j + fr) * C::OUT_PITCH + (32 * i + 8 * q + 4 * fh) * 2) =
          make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
    };
    if constexpr (GRAD) {
      // G = (softmax - [class of the token]) scale, in bf16; zero outside the classes and behind the last token.  A factor that all tokens
      // share is left to the products of G: without it the -1 for the class of a token that the model knows nothing about is exact in
      // bf16, while the same factor on all of them is the same rounding error for all, which no sum averages out.  dh and dw of 8028 tokens
      // against 32000 classes are 0.19 % off in the 2-norm (0.166 % is the rounding of the results themselves, 0.096 % that of G), and were
      // 0.24 to 0.32 % off with 1 / 8028 inside G.
      auto leave = [&](int part) {                      // of all lanes: what `put` has laid out
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int r0 = 0; r0 < C::WN; r0 += RPI) {
          const int r = r0 + late / CPR, c = late % CPR;
          const uint4 v = *reinterpret_cast<const uint4*>(tile + r * C::OUT_PITCH + c * 16);
          bf16_t* to = g.G + (n0 + wn * C::WN + r) * ldg + (int64_t)part * z.piece + m0 + wm * C::WM + c * 8;
          *reinterpret_cast<uint4*>(to) = v;
        }
      };
      auto softmax = [&](float v, float lse) { return __builtin_amdgcn_exp2f((v - lse) * 1.4426950408889634f); };
      if (MODE == XG_GRAD && m0 + BT <= M && n0 + BT <= N && !g.scale) {
        // Straight through, no accumulator is written: the entry of a token's class, which few tiles have, is put over the others in LDS.
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
          const float lse = tok_lse[j];
#pragma unroll
          for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              put(i, j, q, softmax(acc[i][j][4 * q], lse), softmax(acc[i][j][4 * q + 1], lse), softmax(acc[i][j][4 * q + 2], lse),
                  softmax(acc[i][j][4 * q + 3], lse));
          const int rel = tok_class[j] - (int)z.class0 - m0 - wm * C::WM;              // row of the wavefront's tile that is the class
          if (__any(rel >= 0 && rel < C::WM)) {
            const int mine = rel - 4 * fh;
            float at_class = 0.0f;
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r) at_class = mine == 32 * i + 8 * (r >> 2) + (r & 3) ? acc[i][j][r] : at_class;
            asm volatile("" ::: "memory");
            if (mine >= 0 && mine < C::WM && !(mine & 4))
              *reinterpret_cast<bf16_t*>(tile + (32 * j + fr) * C::OUT_PITCH + rel * 2) = from_f32<bf16_t>(softmax(at_class, lse) - 1.0f);
          }
        }
        leave(0);
      } else {
        const int m_left = M - mw;
        auto entry = [&](int i, int j, int r) {
          const int at = 32 * i + 8 * (r >> 2) + (r & 3);
          float p = softmax(acc[i][j][r], tok_lse[j]);
          p -= tok_class[j] - (int)z.class0 - mw == at ? 1.0f : 0.0f;
          return at < m_left && nw + 32 * j < N ? p * tok_scale[j] : 0.0f;           // a repeated class or token may be anything
        };
        if constexpr (MODE == XG_GRAD) {
#pragma unroll
          for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
              for (int q = 0; q < 4; ++q) put(i, j, q, entry(i, j, 4 * q), entry(i, j, 4 * q + 1), entry(i, j, 4 * q + 2), entry(i, j, 4 * q + 3));
          leave(0);
        } else {
#pragma unroll
          for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[i][j][r] = entry(i, j, r);
#pragma unroll
          for (int part = 0; part < 3; ++part) {
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
              for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                  floatx16_t& v = acc[i][j];
                  put(i, j, q, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
#pragma unroll
                  for (int e = 4 * q; e < 4 * q + 4 && part < 2; ++e) {
                    const float head = __uint_as_float(pack_bf16x2(v[e], v[e]) << 16);
                    v[e] = fabsf(head) < INFINITY ? v[e] - head : 0.0f;
                  }
                }
            leave(part);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          }
        }
      }
    } else {
      // dH: the pieces are added up in acc, the last one leaves for the output.  Slices, and logits, leave for acc in any case, and are
      // joined later.
      float* part = g.acc + (int64_t)slice * N * M;
      const bool add = MODE == XG_DH && g.piece > 0;
      const bool to_acc = MODE == XG_PART || nslice > 1 || (MODE == XG_DH && z.class0 + z.piece < g.pieces.V);
      char* const out = (char*)g.out + (MODE == XG_DW ? z.class0 * g.ldo * (g.out_dtype == EFQAT_F32 ? 4 : 2) : 0);
      auto row_of = [&](int n) -> int64_t { return MODE == XG_DH ? g.rows[n] : n; };
      if constexpr (MODE != XG_PART) {
      const float factor = (g.factor ? g.factor[0] : 1.0f) / (g.mean && valid > 0 ? (float)valid : 1.0f);
      if (g.factor || g.mean) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
          for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] *= factor;
      }
      }
      if (add || to_acc || g.out_dtype == EFQAT_F32) {
#pragma unroll
        for (int j = 0; j < C::TN; ++j) {
          const int n = nw + 32 * j;
          if (n >= N) continue;
          const int64_t row = to_acc ? n : row_of(n);
#pragma unroll
          for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int m = m_of(i, 4 * q), left = M - m;
              if (left <= 0) continue;
              float v[4];
              typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
              if (add) {
                const float* from = part + (int64_t)n * M + m;
                if (left >= 4) {
                  const vec o = *reinterpret_cast<const vec*>(from);
#pragma unroll
                  for (int e = 0; e < 4; ++e) v[e] += o[e];
                } else {
#pragma unroll
                  for (int e = 0; e < 3; ++e)
                    if (e < left) v[e] += from[e];
                }
              }
              if (to_acc || g.out_dtype == EFQAT_F32) {
                float* to = to_acc ? part + row * M + m : (float*)out + row * g.ldo + m;
                if (left >= 4) {
                  vec o;
#pragma unroll
                  for (int e = 0; e < 4; ++e) o[e] = v[e];
                  *reinterpret_cast<vec*>(to) = o;
                } else {
#pragma unroll
                  for (int e = 0; e < 3; ++e)
                    if (e < left) to[e] = v[e];
                }
              } else {
                bf16_t* to = (bf16_t*)out + row * g.ldo + m;
                typedef uint32_t pair __attribute__((ext_vector_type(2), aligned(2)));
                if (left >= 4) {
                  *reinterpret_cast<pair*>(to) = pair{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                } else {
#pragma unroll
                  for (int e = 0; e < 3; ++e)
                    if (e < left) to[e] = from_f32<bf16_t>(v[e]);
                }
              }
            }
        }
      } else {
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
          for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) put(i, j, q, acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int r0 = 0; r0 < C::WN; r0 += RPI) {
          const int r = r0 + late / CPR, c = late % CPR;
          const int n = n0 + wn * C::WN + r, m = m0 + wm * C::WM + c * 8;
          const uint4 v = *reinterpret_cast<const uint4*>(tile + r * C::OUT_PITCH + c * 16);
          const int left = n < N ? M - m : 0;
          if (left > 0) {
            bf16_t* to = (bf16_t*)out + row_of(n) * g.ldo + m;
            if (left >= 8) {
              Raw8<bf16_t> o;
              o.a[0] = v.x; o.a[1] = v.y; o.a[2] = v.z; o.a[3] = v.w;
              o.store(to);
            } else {
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 7; ++e)
                if (e < left) to[e] = (bf16_t)(w[e >> 1] >> (16 * (e & 1)));
            }
          }
        }
      }
    }
  }
#endif
}

// A launch has at most as many blocks as the chip holds; they walk the tiles that there are (an empty block is not free: it waits for
// a CU's LDS like the others).
template <int BT, XentMode MODE>
__global__ __launch_bounds__(XentCfg<BT>::THREADS) void k_xent_gemm(const XentGemmArgs g) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int valid = g.n_valid[0];
  const XentShape z(g, MODE, valid);
  if (z.classes == 0) return;
  const XentTiles t(g, z, MODE, BT);
  const int total = t.total();
  for (int bid = blockIdx.x; bid < total; bid += gridDim.x) {
    xent_gemm_block<BT, MODE>(g, z, t, valid, bid, smem);
    __syncthreads();
  }
#endif
}

// Which tiles of the second product a block takes in a launch of `grid` blocks, whose first `first` have one of the first product's: the
// blocks that have none take `others` each, the rest is shared among those that do.  Blocks and tiles go by eights: a tile stays on the
// XCD whose neighbours it has.
struct XentShare {
  int head, tail, others, last;   // blocks that have (rounded up), that do not; tiles of each of the latter; tiles from which the former share
  // a, b: K stages of a tile of the first and the second product
  __device__ __forceinline__ XentShare(int first, int second, int a, int b, int grid) {
    head = (first + 7) / 8 * 8;
    head = head < grid ? head : grid;
    tail = grid - head;
    others = 0;
    if (tail > 0) {
      const int most = (second + tail - 1) / tail;
      int best = INT32_MAX;
      for (int q = most; q >= 0 && q > most - 8; --q) {
        const int rest = second - q * tail, each = rest > 0 ? (rest + head - 1) / (head > 0 ? head : 1) : 0;
        const int cost = max(q * b, a + each * b);
        if (head == 0 && rest > 0) break;
        if (cost < best) { best = cost; others = q; }
      }
    }
    last = min(second, others * tail);
  }
};

// Both products of G in one grid: neither has to wait for the other's last, partly filled round.  They have as many operations, so dH's
// contraction is cut for half of the blocks, and the others begin with dW: 1843 tokens of width 768 against 30522 classes backward 316 ->
// 296 us (against slices of dH for all blocks, with every block's share of dW on top), 1024 of 1024 against 4096 66 -> 56.
template <int BT>
__global__ __launch_bounds__(XentCfg<BT>::THREADS) void k_xent_gemm_pair(const XentGemmArgs h, const XentGemmArgs w) {
#if defined(__HIP_DEVICE_COMPILE__)
  extern __shared__ __attribute__((aligned(16))) char smem[];
  const int valid = h.n_valid[0];
  const XentShape zh(h, XG_DH, valid), zw(w, XG_DW, valid);
  if (zh.classes == 0) return;
  const XentTiles th(h, zh, XG_DH, BT), tw(w, zw, XG_DW, BT);
  const int first = th.total(), second = tw.total(), grid = gridDim.x, block = blockIdx.x;
  for (int bid = block; bid < first; bid += grid) {
    xent_gemm_block<BT, XG_DH>(h, zh, th, valid, bid, smem);
    __syncthreads();
  }
  // tiles begin .. end - 1 of dW in steps
  int begin = block, end = second, step = grid;
  if (first <= grid) {
    const XentShare share(first, second, zh.nks * h.segments / th.slices, zw.nks * w.segments / tw.slices, grid);
    const bool tail = block >= share.head;
    begin = tail ? block - share.head : share.last + block;
    end = tail ? share.last : second;
    step = tail ? share.tail : share.head;
  } else {
    begin = (block + grid - first % grid) % grid;     // where the first product's last round ends
  }
  for (int bid = begin; bid < end; bid += step) {
    xent_gemm_block<BT, XG_DW>(w, zw, tw, valid, bid, smem);
    __syncthreads();
  }
#endif
}

}  // namespace efqat
