// Softmax cross entropy of z = h w^T over a large vocabulary, and its gradients, without keeping z:
//
//   loss_t = lse_t - z_t[class of t],  lse_t = log sum_v exp(z_tv)
//   G = (exp(z - lse) - [v = class of t]) scale_t,   dh = G w,   dw = G^T h
//
// Forward: one product whose epilogue keeps the largest logit and the sum of exponentials of every token and tile of classes
// (8 bytes for 256 logits), joined by a second pass.  Backward: the classes in pieces; a piece's logits are formed again, leave as
// G in bf16 (a buffer that the last-level cache holds) and are multiplied by w and by h.  G in fewer bits than 32 is what lets both
// products run on the matrix cores at their bf16 rate, like the operands; its rounding is 0.10 % of dh and dw in the 2-norm, that of the
// results themselves 0.17 %.  fp32 operands, and then G too, are three bf16 parts: 24 bits.
// Few tiles of many stages: the logits' contraction is cut over the blocks, and the softmax follows the join of the slices.
//
// 8 T D V operations of a training step are products on the matrix cores and bound it; with few tokens, reading w does.  bf16, 8192
// tokens of width 4096 against 32000 classes, 98 % of them with one: 6.6 ms forward and backward, 1.28 POP/s.  12288 of width 768 against
// 30522, 15 % of them with one: 0.40 ms, 0.87 POP/s.  One token of width 4096: 74 us forward, of which 50 are w at 5.2 TB/s.
//
// Tokens without a class (ignored, or a class outside [0, V)) take no part: the rows that do are counted and copied together
// first, on the device, and every grid is cut to their number there.  What an ignored row holds - NaN included - touches nothing.
#include "gemm_xent.hpp"

#include <algorithm>

namespace efqat {

// ---- tokens that have a class: their rows, classes and scales by slot (few tokens: see xent_few_rows)
struct XentRowsArgs {
  const int64_t* targets;
  int64_t T, V, ignore;
  int32_t *rows, *target, *n_valid, *n_out;           // n_out: the caller's count, nullable
  float *loss, *lse;                                  // forward: zero for the other tokens (loss: nullable)
  // backward: log-sum-exp of the tokens and, where every loss has a gradient of its own, that
  const float *lse_in, *dloss;
  float *slot_lse, *slot_scale;                       // slot_scale: nullable
  const int32_t* counts;                              // NULL, or of every 2048 tokens, those with a class
};
constexpr int kXentOwn = 2;                           // tokens of a thread of k_xent_rows
constexpr int kXentBlock = kXentOwn * 1024;
// tokens with a class among a block's
__global__ __launch_bounds__(1024) void k_xent_count(const int64_t* __restrict__ targets, int64_t T, int64_t V, int64_t ignore,
                                                     int32_t* __restrict__ counts) {
  __shared__ int count[16];
  const int64_t t = (int64_t)blockIdx.x * kXentBlock + threadIdx.x;
  int n = 0;
#pragma unroll
  for (int i = 0; i < kXentOwn; ++i) {
    const int64_t c = t + i * 1024 < T ? targets[t + i * 1024] : -1;
    n += __popcll(__ballot(c >= 0 && c < V && c != ignore));
  }
  if ((threadIdx.x & 63) == 0) count[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) n += count[w];
    counts[blockIdx.x] = n;
  }
}
// A block places 2048 tokens: it counts those with a class among all tokens before its own (eight reads in flight a lane), then ranks its
// own by ballots, so that slots are in the order of the tokens and every access is of neighbours.  One block for all took 9 us for 12288
// tokens.  What is read grows with the square of the tokens: from kXentMany on, the blocks' counts are taken first.
__global__ __launch_bounds__(1024) void k_xent_rows(const XentRowsArgs g) {
  __shared__ int earlier[16], count[kXentOwn * 16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t t0 = (int64_t)blockIdx.x * kXentBlock, t = t0 + threadIdx.x;
  auto has_class = [&](int64_t c) { return c >= 0 && c < g.V && c != g.ignore; };
  int64_t c[kXentOwn];
#pragma unroll
  for (int i = 0; i < kXentOwn; ++i) c[i] = t + i * 1024 < g.T ? g.targets[t + i * 1024] : -1;
  int before = 0;
  if (g.counts) {
    for (int64_t u = threadIdx.x; u < (int64_t)blockIdx.x; u += 1024) before += g.counts[u];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) before += __shfl_xor(before, off);
  }
  for (int64_t u0 = 0; u0 < t0 && !g.counts; u0 += 8 * 1024) {
    int64_t v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int64_t u = u0 + i * 1024 + threadIdx.x;
      v[i] = g.targets[u < t0 ? u : threadIdx.x];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) before += __popcll(__ballot(u0 + i * 1024 < t0 && has_class(v[i])));
  }
  uint64_t who[kXentOwn];
#pragma unroll
  for (int i = 0; i < kXentOwn; ++i) {
    who[i] = __ballot(has_class(c[i]));
    if (lane == 0) count[i * 16 + wave] = __popcll(who[i]);
  }
  if (lane == 0) earlier[wave] = before;
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) total += earlier[w];
#pragma unroll
  for (int i = 0; i < kXentOwn; ++i) {
    int slot = total + __popcll(who[i] & ((UINT64_C(1) << lane) - 1));
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      slot += w < wave ? count[i * 16 + w] : 0;
      total += count[i * 16 + w];
    }
    const int64_t ti = t + i * 1024;
    if (who[i] >> lane & 1) {
      g.rows[slot] = (int32_t)ti;
      g.target[slot] = (int32_t)c[i];
      if (g.slot_lse) g.slot_lse[slot] = g.lse_in[ti];
      if (g.slot_scale) g.slot_scale[slot] = g.dloss[ti];
    } else if (ti < g.T) {
      if (g.loss) g.loss[ti] = 0.0f;
      if (g.lse) g.lse[ti] = 0.0f;
    }
  }
  if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 0) {
    g.n_valid[0] = total;
    if (g.n_out) g.n_out[0] = total;
  }
}

// ---- operands in bf16, in rows of whole K stages -> dst [row][PARTS][pitch], zeros behind the columns and the rows.  Tokens: the rows
// rows[] of the slots that exist; backward, rows of dh without a class are cleared on the way.  Classes: those of a piece.
struct XentStageArgs {
  const void* src;
  int64_t ld;
  int64_t cols, pitch;                                // pitch: cols rounded up to 64
  const int32_t *rows, *n_valid;                      // rows NULL: classes
  XentPieces pieces;
  int piece;
  int64_t dst_rows;                                   // most rows of dst
  bf16_t* dst;
  const int64_t* targets;                             // with clear
  int64_t T, V, ignore;
  void* clear;
  int64_t ld_clear;
};
// What k_xent_rows does, by every block of 256 threads for itself, for up to kXentFew tokens: the rows by slot, and their number.  The
// block that writes leaves all of it in memory for the kernels that follow.
constexpr int kXentFew = 1024;
__device__ __forceinline__ int xent_few_rows(const XentRowsArgs& g, bool writes, int* row_of_slot) {
  __shared__ int count[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t c[4];
  uint64_t who[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = i * 256 + threadIdx.x;
    c[i] = t < g.T ? g.targets[t] : -1;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    who[i] = __ballot(c[i] >= 0 && c[i] < g.V && c[i] != g.ignore);
    if (lane == 0) count[i * 4 + wave] = __popcll(who[i]);
  }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = i * 256 + threadIdx.x;
    int slot = __popcll(who[i] & ((UINT64_C(1) << lane) - 1)) + total;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      slot += w < wave ? count[i * 4 + w] : 0;
      total += count[i * 4 + w];
    }
    if (who[i] >> lane & 1) {
      row_of_slot[slot] = t;
      if (writes) {
        g.rows[slot] = t;
        g.target[slot] = (int32_t)c[i];
        if (g.slot_lse) g.slot_lse[slot] = g.lse_in[t];
        if (g.slot_scale) g.slot_scale[slot] = g.dloss[t];
      }
    } else if (writes && t < g.T) {
      if (g.loss) g.loss[t] = 0.0f;
      if (g.lse) g.lse[t] = 0.0f;
    }
  }
  if (writes && threadIdx.x == 0) {
    g.n_valid[0] = total;
    if (g.n_out) g.n_out[0] = total;
  }
  __syncthreads();
  return total;
}

// tokens (blocks 0 .. first - 1) and classes (the others) in one launch; FEW: it finds the tokens that have a class itself
template <typename T, int PARTS, bool FEW>
__global__ __launch_bounds__(256) void k_xent_stage(const XentStageArgs tokens, int first_blocks, const XentStageArgs classes, const XentRowsArgs few) {
  __shared__ int row_of_slot[FEW ? kXentFew : 1];
  const bool second = (int)blockIdx.x >= first_blocks;
  const XentStageArgs& g = second ? classes : tokens;
  const int64_t block = second ? (int64_t)blockIdx.x - first_blocks : blockIdx.x;
  int valid;
  if constexpr (FEW) valid = xent_few_rows(few, blockIdx.x == 0, row_of_slot);
  else valid = g.n_valid[0];
  // rows behind the last one: zeros up to whole stages, which dW's contraction (tokens) and dH's (classes) read
  int64_t n = valid, first = 0, dst_rows = (n + 63) / 64 * 64;
  if (!g.rows) {
    const int64_t p = g.pieces.size(valid);
    first = p * g.piece;
    n = g.pieces.V - first < p ? g.pieces.V - first : p;
    if (n <= 0) return;
    dst_rows = (n + 63) / 64 * 64;
  }
  // lanes of a row: as many as its chunks of 8 columns, up to a block
  const int chunks = (int)(g.pitch / 8);
  const int lanes = chunks >= 256 ? 256 : chunks > 64 ? 128 : chunks > 32 ? 64 : chunks > 16 ? 32 : chunks > 8 ? 16 : 8;
  const int64_t r = block * (256 / lanes) + threadIdx.x / lanes;
  const int lane = threadIdx.x % lanes;
  if (r < dst_rows) {
    const bool in = r < n;
    const T* src = (const T*)g.src + (in ? (!g.rows ? first + r : FEW ? (int64_t)row_of_slot[r] : (int64_t)g.rows[r]) : 0) * g.ld;
    bf16_t* dst = g.dst + r * PARTS * g.pitch;
    for (int c = lane; c < chunks; c += lanes) {
      const int64_t left = in ? g.cols - 8 * (int64_t)c : 0;
      float v[8];
      load_chunk(src + 8 * c, (int)(left > 8 ? 8 : left)).get(v);
      if constexpr (PARTS == 1) {
        store_chunk(dst + 8 * c, 8, v);
      } else {
        float p[3][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float q[3];
          split3(v[j], q);
#pragma unroll
          for (int k = 0; k < 3; ++k) p[k][j] = q[k];
        }
#pragma unroll
        for (int k = 0; k < 3; ++k) store_chunk(dst + k * g.pitch + 8 * c, 8, p[k]);
      }
    }
  }
  if (g.clear && r < g.T) {
    const int64_t t = g.targets[r];
    if (t < 0 || t >= g.V || t == g.ignore) {
      const float zero[8] = {};
      for (int64_t c = 8 * lane; c < g.cols; c += 8 * lanes)
        store_chunk((T*)g.clear + r * g.ld_clear + c, (int)std::min<int64_t>(8, g.cols - c), zero);
    }
  }
}

// ---- forward: the tiles of classes joined, TOK tokens a block, by 1024 / TOK groups of lanes that take the tiles in turn.  Up to 64 tokens
// are one block, which takes their mean or sum too: 64 tokens of width 64 against 8000 classes 14.4 us forward, with a launch for the mean
// and four groups of lanes 17.1; 18 of 32 against 68688 (1074 tiles) 36.8 and 46.5.  So are up to 256 of at most 32 tiles (256 of width 64 against 1000 classes 17.2 -> 15.0 us); 256
// tokens 64 at a time took 28.6, not 19.3.
struct XentJoinArgs {
  const float2* part;
  int tiles;
  int64_t slots;
  const int32_t *n_valid, *rows;
  const float* target_logit;
  float *lse, *loss, *slot_loss;                      // loss of the tokens by row, or by slot (each nullable)
  float* total;                                       // of all tokens: one block, or NULL
  int mean;
};
template <int TOK>
__global__ __launch_bounds__(1024) void k_xent_join(const XentJoinArgs g) {
  constexpr int GROUPS = 1024 / TOK, ROWS = TOK < 64 ? 16 : GROUPS;
  __shared__ float2 red[ROWS][TOK];
  __shared__ double sums[TOK < 64 ? 1 : TOK / 64];
  const int lane = threadIdx.x % TOK, grp = threadIdx.x / TOK, wave = threadIdx.x >> 6;
  const int valid = g.n_valid[0];
  if ((int)blockIdx.x * TOK >= valid && !g.total) return;
  const int n = blockIdx.x * TOK + lane;
  float top = -INFINITY, sum = 0.0f;
  auto join = [&](float2 o) {
    const float t = fmaxf(top, o.x), b = t == -INFINITY ? 0.0f : t;
    sum = sum * __builtin_amdgcn_exp2f((top - b) * 1.4426950408889634f) + o.y * __builtin_amdgcn_exp2f((o.x - b) * 1.4426950408889634f);
    top = t;
  };
  if (n < valid) {
    int i = grp;
    for (; i + 7 * GROUPS < g.tiles; i += 8 * GROUPS) {
      float2 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = g.part[(i + u * GROUPS) * g.slots + n];
#pragma unroll
      for (int u = 0; u < 8; ++u) join(v[u]);
    }
    for (; i < g.tiles; i += GROUPS) join(g.part[i * g.slots + n]);
  }
#pragma unroll
  for (int o = TOK; o < 64; o <<= 1) {                // the groups of a wavefront
    const float2 other = make_float2(__shfl_xor(top, o), __shfl_xor(sum, o));
    join(other);
  }
  if ((threadIdx.x & 63) < TOK) red[TOK < 64 ? wave : grp][lane] = make_float2(top, sum);
  __syncthreads();
  double total = 0.0;
  if (threadIdx.x < TOK && n < valid) {
#pragma unroll
    for (int i = 1; i < ROWS; ++i) join(red[i][lane]);
    const float l = top + logf(sum), d = l - g.target_logit[n];
    const int row = g.rows[n];
    g.lse[row] = l;
    if (g.loss) g.loss[row] = d;
    if (g.slot_loss) g.slot_loss[n] = d;
    total = (double)d;
  }
  if (g.total) {
    total = wave_sum(total);
    if constexpr (TOK > 64) {
      if (threadIdx.x < TOK && (threadIdx.x & 63) == 0) sums[wave] = total;
      __syncthreads();
      total = 0.0;
#pragma unroll
      for (int i = 0; i < TOK / 64; ++i) total += sums[i];
    }
    if (threadIdx.x == 0) g.total[0] = valid == 0 ? 0.0f : (float)(g.mean ? total / valid : total);
  }
}

// ---- logits whose contraction was cut: the slices added in their order.  Forward: a token a block, its log-sum-exp and loss.
struct XentLogitsArgs {
  XentGemmArgs gemm;              // of the product that made them
  int bt;
  const int32_t* rows;
  float *lse, *loss, *slot_loss;                      // forward; loss of the tokens by row, or by slot
};
// 4 logits of a token from class m on, of which n exist (the others: -inf)
__device__ __forceinline__ void xent_sum_slices(const float* part, int64_t slice, int slices, int n, float (&v)[4]) {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = 0.0f;
  if (n >= 4) {
    for (int k = 0; k < slices; k += 4) {             // four loads in flight
      vec o[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) o[u] = *reinterpret_cast<const vec*>(part + (k + u < slices ? k + u : k) * slice);
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += k + u < slices ? o[u][e] : 0.0f;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (e < n)
        for (int k = 0; k < slices; ++k) v[e] += part[k * slice + e];
      else
        v[e] = -INFINITY;
    }
  }
}
template <int THREADS>
__global__ __launch_bounds__(THREADS) void k_xent_logits_lse(const XentLogitsArgs g) {
  constexpr int WAVES = THREADS / 64;
  __shared__ float2 red[WAVES];
  const int valid = g.gemm.n_valid[0], lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const XentShape z(g.gemm, XG_PART, valid);
  const int slices = XentTiles(g.gemm, z, XG_PART, g.bt).slices;
  const int64_t slice = (int64_t)z.N * z.M;
  for (int n = blockIdx.x; n < valid; n += gridDim.x) {
    const float* row = g.gemm.acc + (int64_t)n * z.M;
    const int cls = g.gemm.target[n];
    float top = -INFINITY, sum = 0.0f, at_class = -INFINITY;
    auto join = [&](float t2, float s2) {
      const float t = fmaxf(top, t2), b = t == -INFINITY ? 0.0f : t;
      sum = sum * __builtin_amdgcn_exp2f((top - b) * 1.4426950408889634f) + s2 * __builtin_amdgcn_exp2f((t2 - b) * 1.4426950408889634f);
      top = t;
    };
    for (int m = 4 * threadIdx.x; m < z.M; m += 4 * THREADS) {
      float v[4];
      xent_sum_slices(row + m, slice, slices, z.M - m, v);
      const float t = fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), b = t == -INFINITY ? 0.0f : t;
      float s = 0.0f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s += __builtin_amdgcn_exp2f((v[e] - b) * 1.4426950408889634f);
        at_class = m + e == cls ? v[e] : at_class;
      }
      join(t, s);
    }
    // the one lane that met the class knows its logit
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const float t2 = __shfl_xor(top, o), s2 = __shfl_xor(sum, o);
      join(t2, s2);
    }
    if (lane == 0) red[wave] = make_float2(top, sum);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float2 o = red[i];
      if (i == 0) { top = o.x; sum = o.y; }
      else join(o.x, o.y);
    }
    const float l = top + logf(sum);
    if (cls >> 2 == (cls >> 2) / THREADS * THREADS + (int)threadIdx.x) {
      const int r = g.rows[n];
      g.lse[r] = l;
      if (g.loss) g.loss[r] = l - at_class;
      if (g.slot_loss) g.slot_loss[n] = l - at_class;
    }
    __syncthreads();
  }
}
// Backward: G from them, zeros up to whole stages of classes and tokens.  Chunks of 8 classes.
__global__ __launch_bounds__(256) void k_xent_logits_grad(const XentLogitsArgs g) {
  const int valid = g.gemm.n_valid[0];
  const XentShape z(g.gemm, XG_PART, valid);
  const int slices = XentTiles(g.gemm, z, XG_PART, g.bt).slices;
  const int64_t slice = (int64_t)z.N * z.M;
  const int parts = g.gemm.segments == 6 ? 3 : 1;
  const int64_t ldg = (int64_t)parts * z.piece;
  const uint32_t per_row = (uint32_t)(z.M + 63) / 64 * 8;
  const int64_t all = (int64_t)((z.N + 63) / 64 * 64) * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
    const int n = (int)(i / per_row), m = (int)(i - (int64_t)n * per_row) * 8;
    float v[8] = {};
    if (n < z.N && m < z.M) {
      const float lse = g.gemm.lse[n], scale = g.gemm.scale ? g.gemm.scale[n] : 1.0f;
      const int cls = g.gemm.target[n] - m;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        float x[4];
        xent_sum_slices(g.gemm.acc + (int64_t)n * z.M + m + 4 * h, slice, slices, z.M - m - 4 * h, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = __builtin_amdgcn_exp2f((x[e] - lse) * 1.4426950408889634f);
          v[4 * h + e] = m + 4 * h + e < z.M ? (cls == 4 * h + e ? p - 1.0f : p) * scale : 0.0f;
        }
      }
    }
    bf16_t* to = g.gemm.G + n * ldg + m;
    for (int part = 0; part < parts; ++part) {
      store_chunk(to + (int64_t)part * z.piece, 8, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float head = __uint_as_float(pack_bf16x2(v[e], v[e]) << 16);
        v[e] = fabsf(head) < INFINITY ? v[e] - head : 0.0f;
      }
    }
  }
}

// mean or sum over the tokens, in double precision
__global__ __launch_bounds__(1024) void k_xent_reduce_loss(const float* __restrict__ slot_loss, const int32_t* __restrict__ n_valid, int mean,
                                                           float* __restrict__ loss) {
  __shared__ double red[16];
  const int n = n_valid[0];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 4096) {       // four loads in flight
    float v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = slot_loss[i + 1024 * u < n ? i + 1024 * u : i];
#pragma unroll
    for (int u = 0; u < 4; ++u) s += i + 1024 * u < n ? (double)v[u] : 0.0;
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += red[i];
    loss[0] = n == 0 ? 0.0f : (float)(mean ? s / n : s);
  }
}

// slices of K of a product of G added in their order; nothing where there is one (the product wrote its output itself).  dH: after the
// last piece.
template <typename T, XentMode MODE>
__device__ __forceinline__ void xent_join_slices(const XentGemmArgs& g, int bt) {
  const int valid = g.n_valid[0];
  const XentShape z(g, MODE, valid);
  if (MODE == XG_DW && z.classes == 0) return;
  const int nslice = xent_split(z.split_tiles(bt), z.split_stages, g.segments, g.split_blocks);
  if (nslice <= 1) return;
  const int64_t all = (int64_t)z.N * z.M, chunks = (all + 7) / 8;
  T* const out = (T*)g.out + (MODE == XG_DW ? z.class0 * g.ldo : 0);
  auto row_of = [&](int64_t n) -> int64_t { return MODE == XG_DH ? g.rows[n] : n; };
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
    const int64_t at = i * 8;
    const int n8 = (int)std::min<int64_t>(8, all - at);
    float s[8] = {};
    int k = 0;
    for (; k + 4 <= nslice; k += 4) {                 // four loads in flight
      Raw8<float> r[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) r[u] = load_chunk(g.acc + (k + u) * all + at, n8);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float v[8];
        r[u].get(v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += v[j];
      }
    }
    for (; k < nslice; ++k) {
      float v[8];
      load_chunk(g.acc + k * all + at, n8).get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
    const int64_t n = at / z.M, m = at - n * z.M;
    if (m + 8 <= z.M) {
      store_chunk(out + row_of(n) * g.ldo + m, n8, s);
    } else {                                          // the chunk passes the end of a row
      for (int j = 0; j < n8; ++j) {
        const int64_t nj = (at + j) / z.M, mj = at + j - nj * z.M;
        out[row_of(nj) * g.ldo + mj] = from_f32<T>(s[j]);
      }
    }
  }
}

// dH (blocks of y = 0) and dW (y = 1), those that are asked for
template <typename T>
__global__ __launch_bounds__(256) void k_xent_join_slices(const XentGemmArgs h, int bt_h, const XentGemmArgs w, int bt_w) {
  if (blockIdx.y == 0 && h.out) xent_join_slices<T, XG_DH>(h, bt_h);
  if (blockIdx.y == 1 && w.out) xent_join_slices<T, XG_DW>(w, bt_w);
}

// ---- plans
// Tokens from which on the blocks' counts are taken first: a launch more, 2.5 us of it at work and 3.9 for the places, against 5.8 / 7.8 /
// 12.7 / 199 us in one launch of 12288 / 32768 / 65536 / 1048576 tokens.
constexpr int64_t kXentMany = INT64_C(1) << 15;
// Elements of G at a time: half of what all classes need, 128 MiB of bf16 at least and 512 MiB at most.  A piece costs five launches and
// a pass over the sums of dh: pieces of 128 / 256 / 512 MiB took 505 / 482 / 476 us for 12288 tokens, one in seven with a class, of
// width 768 against 30522 classes, and 6.77 / 6.73 / 6.66 ms for 8192 of width 4096 against 32000.
constexpr int64_t kXentGradLeast = INT64_C(1) << 26, kXentGradMost = INT64_C(1) << 28;
// K stages (of all products of parts) from which on the logits' contraction is cut, where their tiles are fewer than the blocks that the
// chip holds: the slices leave as fp32 sums and the softmax is a pass of its own over them.  Whole / cut, forward and backward, us: 128 fp32
// tokens of width 1920 against 786 classes (180 stages, 26 tiles) 48 + 72 / 29 + 57, 557 bf16 (of 3712, the host knows no better) of 6400
// against 1408 85 + 122 / 38 + 77, 1024 of 4096 against 4096 62 + 145 / 55 + 141.  It costs where there is one slice after all: all 3712 of
// those tokens 103 + 317 / 115 + 263 (the logits, 64 MiB of fp32 at most, are written and read).  With 24 to 32 stages both take the same (512 bf16 of 2048 against 2000 22 + 43 / 23 + 43).
constexpr int64_t kXentCutStages = 48;
constexpr int64_t kXentStageElems = INT64_C(1) << 26; // most elements of a staged piece of W

struct XentPlan {
  int parts, segments;            // bf16 parts of an operand, products of parts
  int64_t Dp, slots;              // features in whole stages, most token slots in whole tiles
  bool stage_w;
  XentPieces pieces;
  int n_pieces;                   // most there can be
  int64_t grad_elems, stage_rows; // of G, of a staged piece
  int bt, bt_dh, bt_dw;           // tiles of the logits and of the two products
  int blocks, blocks_dh, blocks_dw;
  int64_t grid, grid_dh, grid_dw; // tiles and slices, at most
  bool cut;                       // the logits' contraction may be cut
  bool join_dh, join_dw;          // that of a product of G may
  int64_t acc_z, acc_dh, acc_dw;  // fp32 partial results
};

// Tile of the logits: the largest that gives three CUs in four something to do (of 64: whatever is left).  A larger tile reads its operands
// fewer times, a smaller one leaves fewer CUs idle in the last round.  Width 4096, 32000 classes, forward: 65 tokens by 128 / 64 rows 88 /
// 105 us, 256 by 256 / 128 / 64 125 / 102 / 173 us, 1280 by 256 / 128 324 / 342 us.  Up to 64 tokens take 71 to 74 us, of which reading the
// classes is 50.
static int logits_tile(int64_t T, int64_t V) {
  if (T > 128 && ceil_div(V, 256) * ceil_div(T, 256) >= 192) return 256;
  if (T > 64 && ceil_div(V, 128) * ceil_div(T, 128) >= 128) return 128;
  return 64;
}
// Tile and blocks of a product of G [N][M] over so many stages, by the same rule, with the slices of K that there may be.  The backward
// pass of 256 / 768 / 2048 tokens of width 4096 against 32000 classes: tiles of 256 339 / 635 / 1384 us, of 128 360 / 712 / 1593 us; of 128
// tokens 245 us by tiles of 128, 273 by 64.
static int out_tile(int64_t M, int64_t N, int64_t stages, int* blocks) {
  const int64_t t256 = ceil_div(M, 256) * ceil_div(N, 256), t128 = ceil_div(M, 128) * ceil_div(N, 128);
  if (t256 * std::max<int64_t>(1, stages / 12) >= 192 && N > 128) { *blocks = 256; return 256; }
  if (t128 * std::max<int64_t>(1, stages / 12) >= 128 && N > 64) { *blocks = 512; return 128; }
  *blocks = 256;
  return 64;
}
// most fp32 partial results of such a product: slices times rows, for every number of rows from `fewest` to N
static int64_t out_acc_elems(int64_t M, int64_t fewest, int64_t N, int64_t stages, int segments, int bt, int blocks, bool pieces, bool* join) {
  const int64_t tm = ceil_div(M, bt), most = xent_split(tm * ceil_div(fewest, bt), (int)stages, segments, blocks);
  *join = most > 1;
  if (most <= 1 && !pieces) return 0;
  // slices <= blocks / tiles, so that slices * rows <= blocks * bt / tm; a single slice has all rows
  return std::max(N, std::min(most * N, blocks * (int64_t)bt / tm)) * M;
}

// Classes that the products read as they lie: bf16, in rows of whole 16 bytes.  Others are laid out anew, piece by piece, in both passes: of
// width 1360, 53730 of them, 16 tokens, that takes 97 + 196 us forward and backward instead of 46 + 122 (8192 tokens of width 1000 against
// 32000 1 % less: rows of whole 128 bytes).
static bool xent_direct(int dtype, int64_t D, const void* w, int64_t ldw) {
  return dtype == EFQAT_BF16 && D % 8 == 0 && aligned16(w) && ldw % 8 == 0;
}
static XentPlan xent_plan(int64_t T, int64_t D, int64_t V, int dtype, bool direct, bool backward) {
  XentPlan p = {};
  p.parts = dtype == EFQAT_F32 ? 3 : 1;
  p.segments = dtype == EFQAT_F32 ? 6 : 1;
  p.Dp = round_up(D, 64);
  p.slots = round_up(T, 256);
  p.stage_w = !direct;
  p.pieces.V = (int)V;
  p.pieces.parts = p.parts;
  p.pieces.elems = backward ? (uint32_t)std::min(std::max(p.slots * p.parts * round_up(ceil_div(V, 2), 256), kXentGradLeast), kXentGradMost) : 0;
  p.pieces.cap = (int)round_up(V, 256);
  if (p.stage_w) p.pieces.cap = (int)std::min<int64_t>(p.pieces.cap, std::max<int64_t>(kXentStageElems / (p.Dp * p.parts) / 256 * 256, 1024));
  const int64_t piece = p.pieces.size((int)T), widest = p.pieces.size(0);  // of the most and the fewest tokens
  p.n_pieces = (int)ceil_div(V, piece);
  p.stage_rows = p.stage_w ? widest : 0;
  p.bt = logits_tile(T, std::min(V, piece));
  const int64_t stages = p.Dp / 64 * p.segments, tiles = ceil_div(std::min(V, piece), p.bt) * ceil_div(T, p.bt);
  p.blocks = p.bt == 128 ? 512 : 256;
  p.cut = p.n_pieces == 1 && stages >= kXentCutStages && tiles < p.blocks;
  if (p.cut) {
    bool join;
    p.acc_z = std::max(out_acc_elems(V, 1, T, p.Dp / 64, p.segments, p.bt, p.blocks, false, &join), T * V);
  }
  if (!backward) {
    p.grid = p.cut ? p.blocks : ceil_div(piece, p.bt) * ceil_div(T, p.bt);
    return p;
  }
  // a piece of G: `elems`, or 1024 classes of many tokens, or all classes
  p.grad_elems = std::min(p.slots * p.parts * round_up(V, 256), std::max<int64_t>(p.pieces.elems, p.slots * p.parts * 1024));
  p.grid = std::min(ceil_div(V, p.bt) * ceil_div(T, p.bt), p.grad_elems / p.parts / (p.bt * p.bt) + 1);
  if (p.cut) p.grid = p.blocks;
  p.bt_dh = out_tile(D, T, ceil_div(piece, 64) * p.segments, &p.blocks_dh);
  p.bt_dw = out_tile(D, std::min(V, piece), ceil_div(T, 64) * p.segments, &p.blocks_dw);
  p.grid_dh = std::max<int64_t>(ceil_div(D, p.bt_dh) * ceil_div(T, p.bt_dh), p.blocks_dh);
  p.grid_dw = std::max<int64_t>(ceil_div(D, p.bt_dw) * ceil_div(std::min(V, widest), p.bt_dw), p.blocks_dw);
  p.acc_dh = out_acc_elems(D, 1, T, ceil_div(V, 64), p.segments, p.bt_dh, p.blocks_dh, p.n_pieces > 1, &p.join_dh);
  p.acc_dw = out_acc_elems(D, std::min(V, piece), std::min(V, widest), ceil_div(T, 64), p.segments, p.bt_dw, p.blocks_dw, false, &p.join_dw);
  return p;
}

struct XentWs {
  int32_t *n_valid, *rows, *target, *counts;
  bf16_t *h, *w, *grad;
  float2* part;
  float *target_logit, *slot_loss, *slot_lse, *slot_scale, *acc_z, *acc_dh, *acc_dw;
  size_t bytes;
};
static XentWs xent_ws(void* ws, const XentPlan& p, int64_t T, int64_t V, bool backward) {
  WsCarver c(ws);
  XentWs w = {};
  w.n_valid = (int32_t*)c.take(sizeof(int32_t));
  w.rows = (int32_t*)c.take((size_t)T * sizeof(int32_t));
  w.target = (int32_t*)c.take((size_t)T * sizeof(int32_t));
  if (T >= kXentMany) w.counts = (int32_t*)c.take((size_t)ceil_div(T, kXentBlock) * sizeof(int32_t));
  w.h = (bf16_t*)c.take((size_t)(p.slots * p.parts * p.Dp) * 2);
  if (p.stage_w) w.w = (bf16_t*)c.take((size_t)(p.stage_rows * p.parts * p.Dp) * 2);
  w.acc_z = (float*)c.take((size_t)p.acc_z * sizeof(float));
  if (backward) {
    w.slot_lse = (float*)c.take((size_t)T * sizeof(float));
    w.slot_scale = (float*)c.take((size_t)T * sizeof(float));
    w.grad = (bf16_t*)c.take((size_t)p.grad_elems * 2);
    w.acc_dh = (float*)c.take((size_t)p.acc_dh * sizeof(float));
    w.acc_dw = (float*)c.take((size_t)p.acc_dw * sizeof(float));
  } else {
    w.part = (float2*)c.take((size_t)(ceil_div(V, p.bt) * p.slots) * sizeof(float2));
    w.target_logit = (float*)c.take((size_t)T * sizeof(float));
    w.slot_loss = (float*)c.take((size_t)T * sizeof(float));
  }
  w.bytes = c.off;
  return w;
}

static bool xent_sizes_ok(int64_t T, int64_t D, int64_t V) {
  return T > 0 && D > 0 && V > 0 && T <= INT64_C(1) << 30 && V <= INT64_C(1) << 30 && D <= INT64_C(1) << 20;
}
// of a call whose pointers are not known yet
static size_t xent_bytes(int64_t T, int64_t D, int64_t V, int dtype, bool backward) {
  if (!xent_sizes_ok(T, D, V) || !known_dtype(dtype)) return 256;
  const bool may = xent_direct(dtype, D, nullptr, 0), must = may && D % 64 == 0;
  const size_t as_is = may ? xent_ws(nullptr, xent_plan(T, D, V, dtype, true, backward), T, V, backward).bytes : 0;
  return must ? as_is : std::max(as_is, xent_ws(nullptr, xent_plan(T, D, V, dtype, false, backward), T, V, backward).bytes);
}

template <int BT, XentMode MODE>
static int launch_xent_gemm(const XentGemmArgs& g, int64_t blocks, hipStream_t st) {
  using C = XentCfg<BT>;
  static const hipError_t attr = hipFuncSetAttribute((const void*)k_xent_gemm<BT, MODE>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
  if (attr != hipSuccess) return EFQAT_ERR_HIP;
  return launch((k_xent_gemm<BT, MODE>), dim3((unsigned)std::min<int64_t>(blocks, C::CHIP)), dim3(C::THREADS), C::LDS, st, g);
}
template <XentMode MODE>
static int launch_xent_tile(int bt, const XentGemmArgs& g, int64_t blocks, hipStream_t st) {
  if (bt == 256) return launch_xent_gemm<256, MODE>(g, blocks, st);
  if (bt == 128) return launch_xent_gemm<128, MODE>(g, blocks, st);
  return launch_xent_gemm<64, MODE>(g, blocks, st);
}
template <int BT>
static int launch_xent_pair(const XentGemmArgs& h, const XentGemmArgs& w, int64_t blocks, hipStream_t st) {
  using C = XentCfg<BT>;
  static const hipError_t attr = hipFuncSetAttribute((const void*)k_xent_gemm_pair<BT>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
  if (attr != hipSuccess) return EFQAT_ERR_HIP;
  return launch(k_xent_gemm_pair<BT>, dim3((unsigned)std::min<int64_t>(blocks, C::CHIP)), dim3(C::THREADS), C::LDS, st, h, w);
}

static int launch_rows(XentRowsArgs r, int32_t* counts, hipStream_t st) {
  const dim3 grid((unsigned)ceil_div(r.T, kXentBlock));
  if (counts) EFQAT_TRY(launch(k_xent_count, grid, dim3(1024), 0, st, r.targets, r.T, r.V, r.ignore, counts));
  r.counts = counts;
  return launch(k_xent_rows, grid, dim3(1024), 0, st, r);
}

static int stage_blocks(int64_t rows, int64_t pitch, unsigned* blocks) {
  const int64_t chunks = pitch / 8;
  const int64_t lanes = chunks >= 256 ? 256 : chunks > 64 ? 128 : chunks > 32 ? 64 : chunks > 16 ? 32 : chunks > 8 ? 16 : 8;
  const int64_t n = ceil_div(rows, 256 / lanes);
  if (n > INT32_MAX) return EFQAT_ERR_BAD_SHAPE;
  *blocks = (unsigned)n;
  return EFQAT_OK;
}
// tokens and / or classes (NULL: none).  rows: with up to kXentFew tokens, what would have been k_xent_rows' arguments
static int launch_stage(const XentStageArgs* tokens, const XentStageArgs* classes, const XentRowsArgs* rows, int dtype, hipStream_t st) {
  const XentStageArgs none = {};
  unsigned n_tokens = 0, n_classes = 0;
  if (tokens) EFQAT_TRY(stage_blocks(std::max(tokens->dst_rows, tokens->clear ? tokens->T : 0), tokens->pitch, &n_tokens));
  if (classes) EFQAT_TRY(stage_blocks(classes->dst_rows, classes->pitch, &n_classes));
  if ((int64_t)n_tokens + n_classes > INT32_MAX) return EFQAT_ERR_BAD_SHAPE;
  const dim3 grid(n_tokens + n_classes);
  const XentStageArgs &t = tokens ? *tokens : none, &c = classes ? *classes : none;
  const XentRowsArgs no_rows = {}, &r = rows ? *rows : no_rows;
#define EFQAT_STAGE(E, PARTS, FEW) return launch((k_xent_stage<E, PARTS, FEW>), grid, dim3(256), 0, st, t, (int)n_tokens, c, r)
  if (dtype == EFQAT_F32) { if (rows) EFQAT_STAGE(float, 3, true); EFQAT_STAGE(float, 3, false); }
  if (rows) EFQAT_STAGE(bf16_t, 1, true);
  EFQAT_STAGE(bf16_t, 1, false);
#undef EFQAT_STAGE
}

static XentGemmArgs xent_gemm_args(const XentPlan& p, const XentWs& k, const void* w, int64_t ldw, int64_t D) {
  XentGemmArgs g = {};
  g.W = p.stage_w ? k.w : (const bf16_t*)w;
  g.w_piece = p.stage_w ? 1 : 0;
  g.ldw = p.stage_w ? p.parts * p.Dp : ldw;
  g.H = k.h;
  g.G = k.grad;
  g.Dp = p.Dp;
  g.D = D;
  g.segments = p.segments;
  g.pieces = p.pieces;
  g.n_valid = k.n_valid;
  g.target = k.target;
  g.slots = p.slots;
  return g;
}
static XentStageArgs xent_stage_tokens(const XentPlan& p, const XentWs& k, const void* h, int64_t ldh, int64_t D) {
  XentStageArgs s = {};
  s.src = h; s.ld = ldh; s.cols = D; s.pitch = p.Dp; s.rows = k.rows; s.n_valid = k.n_valid; s.dst_rows = p.slots; s.dst = k.h;
  return s;
}
static XentStageArgs xent_stage_classes(const XentPlan& p, const XentWs& k, const void* w, int64_t ldw, int64_t D) {
  XentStageArgs s = {};
  s.src = w; s.ld = ldw; s.cols = D; s.pitch = p.Dp; s.n_valid = k.n_valid; s.pieces = p.pieces; s.dst_rows = p.stage_rows; s.dst = k.w;
  return s;
}

static int check_xent(const void* h, int64_t ldh, const void* w, int64_t ldw, int dtype, int64_t T, int64_t D, int64_t V,
                      const int64_t* targets, int reduction, const void* ws) {
  // token slots and classes are 32-bit numbers, offsets inside a tile of 256 rows too
  if (!xent_sizes_ok(T, D, V) || ldh < D || ldw < D || ldw > INT64_C(1) << 22) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (reduction != EFQAT_XENT_NONE && reduction != EFQAT_XENT_MEAN && reduction != EFQAT_XENT_SUM) return EFQAT_ERR_BAD_LAYOUT;
  if (!h || !w || !targets || !ws) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(h, dtype) || !aligned_for(w, dtype) || ((uintptr_t)targets % 8) != 0 || ((uintptr_t)ws % 256) != 0)
    return EFQAT_ERR_ALIGNMENT;
  // classes of whole K stages are read as they lie, 16 bytes at a time
  if (dtype == EFQAT_BF16 && D % 64 == 0 && (!aligned16(w) || ldw % 8 != 0)) return EFQAT_ERR_ALIGNMENT;
  return EFQAT_OK;
}

}  // namespace efqat

using namespace efqat;

extern "C" size_t efqat_linear_xent_fwd_workspace_bytes(int64_t T, int64_t D, int64_t V, int dtype) { return xent_bytes(T, D, V, dtype, false); }
extern "C" size_t efqat_linear_xent_bwd_workspace_bytes(int64_t T, int64_t D, int64_t V, int dtype) { return xent_bytes(T, D, V, dtype, true); }

extern "C" int efqat_linear_xent_fwd(const void* h, int64_t ldh, const void* w, int64_t ldw, int dtype, int64_t T, int64_t D, int64_t V,
                                     const int64_t* targets, int64_t ignore_index, int reduction, float* loss, float* lse,
                                     int32_t* n_valid, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_xent(h, ldh, w, ldw, dtype, T, D, V, targets, reduction, ws)) return rc;
  if (!loss || !lse) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(loss) || !aligned4(lse) || !aligned4(n_valid)) return EFQAT_ERR_ALIGNMENT;
  const XentPlan p = xent_plan(T, D, V, dtype, xent_direct(dtype, D, w, ldw), false);
  const XentWs k = xent_ws(ws, p, T, V, false);
  if (ws_bytes < k.bytes) return EFQAT_ERR_WORKSPACE;
  if (std::max({p.grid, p.grid_dh, p.grid_dw}) > INT32_MAX / 2) return EFQAT_ERR_BAD_SHAPE;
  hipStream_t st = (hipStream_t)stream;
  const bool none = reduction == EFQAT_XENT_NONE;

  XentRowsArgs r = {};
  r.targets = targets; r.T = T; r.V = V; r.ignore = ignore_index;
  r.rows = k.rows; r.target = k.target; r.n_valid = k.n_valid; r.n_out = n_valid;
  r.loss = none ? loss : nullptr; r.lse = lse;
  const bool few = T <= kXentFew;
  if (!few) EFQAT_TRY(launch_rows(r, k.counts, st));

  const XentStageArgs tokens = xent_stage_tokens(p, k, h, ldh, D);
  XentStageArgs classes = xent_stage_classes(p, k, w, ldw, D);
  XentGemmArgs g = xent_gemm_args(p, k, w, ldw, D);
  g.part = k.part;
  g.target_logit = k.target_logit;
  for (g.piece = 0; g.piece < p.n_pieces; ++g.piece) {
    classes.piece = g.piece;
    if (p.stage_w || g.piece == 0) EFQAT_TRY(launch_stage(g.piece == 0 ? &tokens : nullptr, p.stage_w ? &classes : nullptr, few && g.piece == 0 ? &r : nullptr, dtype, st));
    if (!p.cut) EFQAT_TRY(launch_xent_tile<XG_LSE>(p.bt, g, p.grid, st));
  }
  const int mean = reduction == EFQAT_XENT_MEAN ? 1 : 0;
  if (p.cut) {
    g.piece = 0;
    g.acc = k.acc_z;
    g.split_blocks = p.blocks;
    EFQAT_TRY(launch_xent_tile<XG_PART>(p.bt, g, p.grid, st));
    const XentLogitsArgs z = {g, p.bt, k.rows, lse, none ? loss : nullptr, none ? nullptr : k.slot_loss};
    EFQAT_TRY(T <= 256 ? launch(k_xent_logits_lse<1024>, dim3((unsigned)T), dim3(1024), 0, st, z)
                       : launch(k_xent_logits_lse<256>, dim3((unsigned)std::min<int64_t>(T, 2048)), dim3(256), 0, st, z));
    if (none) return EFQAT_OK;
    return launch(k_xent_reduce_loss, dim3(1), dim3(1024), 0, st, k.slot_loss, k.n_valid, mean, loss);
  }

  // tiles of a piece are whole but for the last piece's: pieces are multiples of 256 classes
  XentJoinArgs j = {};
  j.part = k.part; j.tiles = (int)ceil_div(V, p.bt); j.slots = p.slots; j.n_valid = k.n_valid; j.rows = k.rows;
  j.target_logit = k.target_logit; j.lse = lse; j.loss = none ? loss : nullptr;
  const bool one = !none && (T <= 64 || (T <= 256 && j.tiles <= 32));
  if (one) { j.total = loss; j.mean = mean; }
  else if (!none) j.slot_loss = k.slot_loss;
  if (T <= 16) EFQAT_TRY(launch(k_xent_join<16>, dim3(1), dim3(1024), 0, st, j));
  else if (T > 64 && one) EFQAT_TRY(launch(k_xent_join<256>, dim3(1), dim3(1024), 0, st, j));
  else EFQAT_TRY(launch(k_xent_join<64>, dim3((unsigned)ceil_div(T, 64)), dim3(1024), 0, st, j));
  if (none || one) return EFQAT_OK;
  return launch(k_xent_reduce_loss, dim3(1), dim3(1024), 0, st, k.slot_loss, k.n_valid, mean, loss);
}

extern "C" int efqat_linear_xent_bwd(const void* h, int64_t ldh, const void* w, int64_t ldw, int dtype, int64_t T, int64_t D, int64_t V,
                                     const int64_t* targets, int64_t ignore_index, int reduction, const float* lse, const float* dloss,
                                     void* dh, int64_t lddh, void* dw, int64_t lddw, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_xent(h, ldh, w, ldw, dtype, T, D, V, targets, reduction, ws)) return rc;
  if ((dh && lddh < D) || (dw && lddw < D)) return EFQAT_ERR_BAD_SHAPE;
  if (!lse || (!dh && !dw)) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(lse) || !aligned4(dloss) || !aligned_for(dh, dtype) || !aligned_for(dw, dtype)) return EFQAT_ERR_ALIGNMENT;
  const XentPlan p = xent_plan(T, D, V, dtype, xent_direct(dtype, D, w, ldw), true);
  const XentWs k = xent_ws(ws, p, T, V, true);
  if (ws_bytes < k.bytes) return EFQAT_ERR_WORKSPACE;
  if (std::max({p.grid, p.grid_dh, p.grid_dw}) > INT32_MAX / 2) return EFQAT_ERR_BAD_SHAPE;
  hipStream_t st = (hipStream_t)stream;

  XentRowsArgs r = {};
  r.targets = targets; r.T = T; r.V = V; r.ignore = ignore_index;
  r.rows = k.rows; r.target = k.target; r.n_valid = k.n_valid;
  const bool own = reduction == EFQAT_XENT_NONE && dloss;          // gradients of the tokens' losses
  r.lse_in = lse; r.slot_lse = k.slot_lse;
  r.dloss = own ? dloss : nullptr; r.slot_scale = own ? k.slot_scale : nullptr;
  const bool few = T <= kXentFew;
  if (!few) EFQAT_TRY(launch_rows(r, k.counts, st));

  XentStageArgs tokens = xent_stage_tokens(p, k, h, ldh, D), classes = xent_stage_classes(p, k, w, ldw, D);
  tokens.targets = targets; tokens.T = T; tokens.V = V; tokens.ignore = ignore_index; tokens.clear = dh; tokens.ld_clear = lddh;
  XentGemmArgs g = xent_gemm_args(p, k, w, ldw, D);
  g.lse = k.slot_lse;
  g.scale = own ? k.slot_scale : nullptr;
  g.factor = own ? nullptr : dloss;
  g.mean = reduction == EFQAT_XENT_MEAN ? 1 : 0;
  g.out_dtype = dtype;
  for (g.piece = 0; g.piece < p.n_pieces; ++g.piece) {
    classes.piece = g.piece;
    if (p.stage_w || g.piece == 0) EFQAT_TRY(launch_stage(g.piece == 0 ? &tokens : nullptr, p.stage_w ? &classes : nullptr, few && g.piece == 0 ? &r : nullptr, dtype, st));
    if (p.cut) {
      XentGemmArgs gz = g;
      gz.acc = k.acc_z;
      gz.split_blocks = p.blocks;
      EFQAT_TRY(launch_xent_tile<XG_PART>(p.bt, gz, p.grid, st));
      const XentLogitsArgs z = {gz, p.bt, nullptr, nullptr, nullptr, nullptr};
      const int64_t chunks = round_up(T, 64) * (round_up(V, 64) / 8);
      EFQAT_TRY(launch(k_xent_logits_grad, dim3((unsigned)std::min<int64_t>(ceil_div(chunks, 256), 2048)), dim3(256), 0, st, z));
    } else {
      EFQAT_TRY(p.parts == 3 ? launch_xent_tile<XG_GRAD3>(p.bt, g, p.grid, st) : launch_xent_tile<XG_GRAD>(p.bt, g, p.grid, st));
    }
    XentGemmArgs gh = g, gw = g;
    gh.split_blocks = p.blocks_dh; gh.acc = k.acc_dh; gh.out = dh; gh.ldo = lddh; gh.rows = k.rows;
    gw.split_blocks = p.blocks_dw; gw.acc = k.acc_dw; gw.out = dw; gw.ldo = lddw;
    if (dh && dw && p.bt_dh == p.bt_dw) {
      const int64_t blocks = p.grid_dh + p.grid_dw;
      gh.split_blocks /= 2;                           // as many operations in each: half of the blocks for dH's slices
      EFQAT_TRY(p.bt_dh == 256   ? launch_xent_pair<256>(gh, gw, blocks, st)
                : p.bt_dh == 128 ? launch_xent_pair<128>(gh, gw, blocks, st)
                                 : launch_xent_pair<64>(gh, gw, blocks, st));
    } else {
      if (dh) EFQAT_TRY(launch_xent_tile<XG_DH>(p.bt_dh, gh, p.grid_dh, st));
      if (dw) EFQAT_TRY(launch_xent_tile<XG_DW>(p.bt_dw, gw, p.grid_dw, st));
    }
    if (!p.join_dh || g.piece < p.n_pieces - 1) gh.out = nullptr;
    if (!p.join_dw) gw.out = nullptr;
    if (gh.out || gw.out) {
      const int64_t most = std::max(gh.out ? T : 0, gw.out ? std::min(V, (int64_t)p.pieces.size(0)) : 0) * D;
      const dim3 grid((unsigned)std::min<int64_t>(ceil_div(most, 8 * 256), 1024), gw.out ? 2 : 1);
      EFQAT_TRY(dtype == EFQAT_F32 ? launch(k_xent_join_slices<float>, grid, dim3(256), 0, st, gh, p.bt_dh, gw, p.bt_dw)
                                   : launch(k_xent_join_slices<bf16_t>, grid, dim3(256), 0, st, gh, p.bt_dh, gw, p.bt_dw));
    }
  }
  return EFQAT_OK;
}
