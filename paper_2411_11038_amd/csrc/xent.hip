// Softmax cross entropy of z = h w^T over a large vocabulary, and its gradients, without keeping z:
//
//   loss_t = lse_t - z_t[class of t],  lse_t = log sum_v exp(z_tv)
//   G = (exp(z - lse) - [v = class of t]) scale_t,   dh = G w,   dw = G^T h
//
// Forward: one product whose epilogue keeps the largest logit and the sum of exponentials of every token and tile of classes
// (8 bytes for 256 logits), joined by a second pass.  Backward: the classes in pieces; a piece's logits are formed again, leave as
// G in bf16 (a buffer that the last-level cache holds) and are multiplied by w and by h.  8 T D V operations of a training step
// are products on the matrix cores and bound it.
//
// Tokens without a class (ignored, or a class outside [0, V)) take no part: the rows that do are counted and copied together
// first, on the device, and every grid is cut to their number there.  What an ignored row holds - NaN included - touches nothing.
#include "gemm_xent.hpp"

#include <algorithm>

namespace efqat {

// ---- tokens that have a class: their rows, classes and scales by slot
struct XentRowsArgs {
  const int64_t* targets;
  int64_t T, V, ignore;
  int32_t *rows, *target, *n_valid, *n_out;           // n_out: the caller's count, nullable
  float *loss, *lse;                                  // forward: zero for the other tokens (loss: nullable)
  // backward: what the loss of a token is multiplied by
  const float *lse_in, *dloss;
  int reduction;
  float *slot_lse, *slot_scale;
};
__global__ __launch_bounds__(1024) void k_xent_rows(const XentRowsArgs g) {
  __shared__ int wave_count[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t per = (g.T + 1023) / 1024;
  const int64_t t0 = threadIdx.x * per, t1 = t0 + per < g.T ? t0 + per : g.T;
  auto has_class = [&](int64_t c) { return c >= 0 && c < g.V && c != g.ignore; };
  int mine = 0;
  for (int64_t t = t0; t < t1; ++t) mine += has_class(g.targets[t]) ? 1 : 0;
  int before = mine;                                  // inclusive scan of the wavefront
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(before, o);
    before += lane >= o ? v : 0;
  }
  if (lane == 63) wave_count[wave] = before;
  __syncthreads();
  int slot = before - mine, total = 0;
#pragma unroll
  for (int w = 0; w < 16; ++w) {
    if (w < wave) slot += wave_count[w];
    total += wave_count[w];
  }
  if (threadIdx.x == 0) {
    g.n_valid[0] = total;
    if (g.n_out) g.n_out[0] = total;
  }
  float scale = 1.0f;
  if (g.slot_scale && g.reduction != EFQAT_XENT_NONE) {
    scale = g.dloss ? g.dloss[0] : 1.0f;
    if (g.reduction == EFQAT_XENT_MEAN) scale /= (float)total;
  }
  for (int64_t t = t0; t < t1; ++t) {
    const int64_t c = g.targets[t];
    if (has_class(c)) {
      g.rows[slot] = (int32_t)t;
      g.target[slot] = (int32_t)c;
      if (g.slot_scale) {
        g.slot_lse[slot] = g.lse_in[t];
        g.slot_scale[slot] = g.reduction == EFQAT_XENT_NONE && g.dloss ? g.dloss[t] : scale;
      }
      ++slot;
    } else {
      if (g.loss) g.loss[t] = 0.0f;
      if (g.lse) g.lse[t] = 0.0f;
    }
  }
}

// ---- operands in bf16, in rows of whole K stages: src rows (by rows[], those of the slots that exist) -> dst [row][PARTS][pitch],
// zeros behind the columns and the rows.  Backward: rows of dh without a class are cleared on the way.
struct XentStageArgs {
  const void* src;
  int64_t ld;
  int64_t cols, pitch;                                // pitch: cols rounded up to 64
  const int32_t *rows, *n_valid;                      // NULL: rows as they lie, n_rows of them
  int64_t n_rows, dst_rows;
  bf16_t* dst;
  const int64_t* targets;                             // with clear
  int64_t T, V, ignore;
  void* clear;
  int64_t ld_clear;
};
template <typename T, int PARTS>
__global__ __launch_bounds__(256) void k_xent_stage(const XentStageArgs g) {
  const int64_t n = g.n_valid ? g.n_valid[0] : g.n_rows;
  // lanes of a row: as many as its chunks of 8 columns, up to a block
  const int chunks = (int)(g.pitch / 8);
  const int lanes = chunks >= 256 ? 256 : chunks > 64 ? 128 : chunks > 32 ? 64 : chunks > 16 ? 32 : chunks > 8 ? 16 : 8;
  const int64_t r = (int64_t)blockIdx.x * (256 / lanes) + threadIdx.x / lanes;
  const int lane = threadIdx.x % lanes;
  if (r < g.dst_rows) {
    const bool in = r < n;
    const T* src = (const T*)g.src + (in ? (g.rows ? (int64_t)g.rows[r] : r) : 0) * g.ld;
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

// ---- forward: the tiles of classes joined, 64 tokens a block, four groups of tiles
__global__ __launch_bounds__(256) void k_xent_join(const float2* __restrict__ part, int tiles, int slots, const int32_t* __restrict__ n_valid,
                                                   const int32_t* __restrict__ rows, const float* __restrict__ target_logit,
                                                   float* __restrict__ lse, float* __restrict__ loss, float* __restrict__ slot_loss) {
  __shared__ float2 red[4][64];
  const int lane = threadIdx.x & 63, grp = threadIdx.x >> 6;
  const int n = blockIdx.x * 64 + lane;
  const int valid = n_valid[0];
  if ((int)blockIdx.x * 64 >= valid) return;
  float top = -INFINITY, sum = 0.0f;
  auto join = [&](float2 o) {
    const float t = fmaxf(top, o.x), b = t == -INFINITY ? 0.0f : t;
    sum = sum * __builtin_amdgcn_exp2f((top - b) * 1.4426950408889634f) + o.y * __builtin_amdgcn_exp2f((o.x - b) * 1.4426950408889634f);
    top = t;
  };
  if (n < valid) {
    int i = grp;
    for (; i + 28 < tiles; i += 32) {
      float2 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) v[u] = part[(int64_t)(i + 4 * u) * slots + n];
#pragma unroll
      for (int u = 0; u < 8; ++u) join(v[u]);
    }
    for (; i < tiles; i += 4) join(part[(int64_t)i * slots + n]);
  }
  red[grp][lane] = make_float2(top, sum);
  __syncthreads();
  if (grp != 0 || n >= valid) return;
#pragma unroll
  for (int i = 1; i < 4; ++i) join(red[i][lane]);
  const float l = top + logf(sum), d = l - target_logit[n];
  const int row = rows[n];
  lse[row] = l;
  if (loss) loss[row] = d;
  else slot_loss[n] = d;
}

// mean or sum over the tokens, in double precision
__global__ __launch_bounds__(1024) void k_xent_reduce_loss(const float* __restrict__ slot_loss, const int32_t* __restrict__ n_valid, int mean,
                                                           float* __restrict__ loss) {
  __shared__ double red[16];
  const int n = n_valid[0];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += (double)slot_loss[i];
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

// slices of K of an XG_OUT product added in their order; nothing where there is one (the product wrote its output itself)
template <typename T>
__global__ __launch_bounds__(256) void k_xent_join_slices(const XentGemmArgs g, int bt) {
  const int valid = g.n_valid[0];
  const int N = g.count_n ? valid : g.N, K = g.count_k ? valid : g.K;
  const int nslice = xent_split(g.tiles_m * ((N + bt - 1) / bt), g.count_k ? (K + 63) / 64 : g.split_stages, g.split_blocks);
  if (nslice <= 1) return;
  const int64_t all = (int64_t)N * g.M, chunks = (all + 7) / 8;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < chunks; i += (int64_t)gridDim.x * 256) {
    const int64_t at = i * 8;
    const int n8 = (int)std::min<int64_t>(8, all - at);
    float s[8] = {};
    for (int k = 0; k < nslice; ++k) {
      float v[8];
      load_chunk(g.acc + k * all + at, n8).get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s[j] += v[j];
    }
    const int64_t n = at / g.M, m = at - n * g.M;
    if (m + 8 <= g.M) {
      store_chunk((T*)g.out + (g.rows ? (int64_t)g.rows[n] : n) * g.ldo + m, n8, s);
    } else {                                          // the chunk passes the end of a row
      for (int j = 0; j < n8; ++j) {
        const int64_t nj = (at + j) / g.M, mj = at + j - nj * g.M;
        ((T*)g.out)[(g.rows ? (int64_t)g.rows[nj] : nj) * g.ldo + mj] = from_f32<T>(s[j]);
      }
    }
  }
}

// ---- plans
constexpr int64_t kXentGradElems = INT64_C(1) << 26;  // most elements of G at a time: 128 MiB of bf16, which the last-level cache holds
constexpr int64_t kXentStageElems = INT64_C(1) << 26; // most elements of a staged piece of W

struct XentPlan {
  int parts;                      // bf16 parts of an operand
  int64_t Dp, slots;              // features in whole stages, token slots in whole tiles
  bool stage_w;
  int64_t piece;                  // classes of a piece, a multiple of 256 (one piece: all of them, rounded up)
  int64_t pieces;
  int bt;                         // tile of the logits
  int bt_dh, bt_dw, blocks_dh, blocks_dw;
  int64_t acc_dh, acc_dw;         // fp32 partial results
};

static int logits_tile(int64_t T, int64_t V) {
  if (T > 128 && ceil_div(V, 256) * ceil_div(T, 256) >= 192) return 256;
  if (T > 64 && ceil_div(V, 128) * ceil_div(T, 128) >= 128) return 128;
  return 64;
}
// tile and blocks of an XG_OUT product [N][M] over so many stages
static int out_tile(int64_t M, int64_t N, int64_t stages, int* blocks) {
  const int64_t t256 = ceil_div(M, 256) * ceil_div(N, 256), t128 = ceil_div(M, 128) * ceil_div(N, 128);
  if (t256 * std::max<int64_t>(1, stages / 8) >= 192 && N > 128) { *blocks = 256; return 256; }
  if (t128 * std::max<int64_t>(1, stages / 8) >= 128 && N > 64) { *blocks = 512; return 128; }
  *blocks = 1024;
  return 64;
}
// most fp32 partial results of such a product: slices times rows, for every number of rows up to N
static int64_t out_acc_elems(int64_t M, int64_t N, int64_t stages, int bt, int blocks, bool pieces) {
  const int64_t tm = ceil_div(M, bt);
  const int64_t most = std::max<int64_t>(1, stages / 8);
  // slices <= blocks / tiles, so that slices * rows <= blocks * bt / tm; a single slice has all rows
  int64_t rows = std::min<int64_t>(most * N, std::max<int64_t>(blocks * (int64_t)bt / tm, N));
  if (xent_split((int)std::min<int64_t>(tm, INT32_MAX), (int)std::min<int64_t>(stages, INT32_MAX), blocks) <= 1 && !pieces) rows = 0;
  return rows * M;
}

static XentPlan xent_plan(int64_t T, int64_t D, int64_t V, int dtype, bool backward) {
  XentPlan p = {};
  p.parts = dtype == EFQAT_F32 ? 3 : 1;
  p.Dp = round_up(D, 64);
  p.slots = round_up(T, 256);
  p.stage_w = p.parts == 3 || D % 64 != 0;
  int64_t most = INT64_C(1) << 31;                     // more than there are classes
  if (p.stage_w) most = kXentStageElems / (p.Dp * p.parts);
  if (backward) most = std::min(most, kXentGradElems / (p.slots * p.parts));
  most = std::max<int64_t>(most / 256 * 256, 1024);
  p.pieces = ceil_div(V, most);
  p.piece = round_up(ceil_div(V, p.pieces), 256);
  p.pieces = ceil_div(V, p.piece);
  p.bt = logits_tile(T, std::min(V, p.piece));
  if (backward) {
    const int64_t kv = std::min(V, p.piece);
    p.bt_dh = out_tile(D, T, p.parts == 3 ? kv / 64 * 6 : kv / 64, &p.blocks_dh);
    p.bt_dw = out_tile(D, kv, p.parts == 3 ? T / 64 * 6 : T / 64, &p.blocks_dw);
    p.acc_dh = out_acc_elems(D, T, ceil_div(kv, 64), p.bt_dh, p.blocks_dh, p.pieces > 1);
    p.acc_dw = out_acc_elems(D, kv, ceil_div(T, 64), p.bt_dw, p.blocks_dw, false);
  }
  return p;
}

struct XentWs {
  int32_t *n_valid, *rows, *target;
  bf16_t *h, *w, *grad;
  float2* part;
  float *target_logit, *slot_loss, *slot_lse, *slot_scale, *acc_dh, *acc_dw;
  size_t bytes;
};
static XentWs xent_ws(void* ws, const XentPlan& p, int64_t T, int64_t V, bool backward) {
  WsCarver c(ws);
  XentWs w = {};
  w.n_valid = (int32_t*)c.take(sizeof(int32_t));
  w.rows = (int32_t*)c.take((size_t)T * sizeof(int32_t));
  w.target = (int32_t*)c.take((size_t)T * sizeof(int32_t));
  w.h = (bf16_t*)c.take((size_t)(p.slots * p.parts * p.Dp) * 2);
  if (p.stage_w) w.w = (bf16_t*)c.take((size_t)(p.piece * p.parts * p.Dp) * 2);
  if (backward) {
    w.slot_lse = (float*)c.take((size_t)T * sizeof(float));
    w.slot_scale = (float*)c.take((size_t)T * sizeof(float));
    w.grad = (bf16_t*)c.take((size_t)(p.slots * p.parts * p.piece) * 2);
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

template <int BT, bool ATR, bool BTR, int MODE>
static int launch_xent_gemm(const XentGemmArgs& g, int64_t blocks, hipStream_t st) {
  using C = XentCfg<BT>;
  static const hipError_t attr = hipFuncSetAttribute((const void*)k_xent_gemm<BT, ATR, BTR, MODE>, hipFuncAttributeMaxDynamicSharedMemorySize, C::LDS);
  if (attr != hipSuccess) return EFQAT_ERR_HIP;
  EFQAT_TRY(launch((k_xent_gemm<BT, ATR, BTR, MODE>), dim3((unsigned)blocks), dim3(C::NW * 64), C::LDS, st, g));
  return EFQAT_OK;
}
template <bool ATR, bool BTR, int MODE>
static int launch_xent_tile(int bt, const XentGemmArgs& a, hipStream_t st) {
  XentGemmArgs g = a;
  g.tiles_m = (int)ceil_div(g.M, bt);
  g.tiles_n = (int)ceil_div(g.N, bt);
  int64_t blocks = (int64_t)g.tiles_m * g.tiles_n;
  if (MODE == XG_OUT && g.split_blocks > 0) blocks = std::max<int64_t>(blocks, g.split_blocks);
  if (blocks > INT32_MAX) return EFQAT_ERR_BAD_SHAPE;
  if (bt == 256) return launch_xent_gemm<256, ATR, BTR, MODE>(g, blocks, st);
  if (bt == 128) return launch_xent_gemm<128, ATR, BTR, MODE>(g, blocks, st);
  return launch_xent_gemm<64, ATR, BTR, MODE>(g, blocks, st);
}

static int stage_blocks(int64_t rows, int64_t pitch, unsigned* blocks) {
  const int64_t chunks = pitch / 8;
  const int64_t lanes = chunks >= 256 ? 256 : chunks > 64 ? 128 : chunks > 32 ? 64 : chunks > 16 ? 32 : chunks > 8 ? 16 : 8;
  const int64_t n = ceil_div(rows, 256 / lanes);
  if (n > INT32_MAX) return EFQAT_ERR_BAD_SHAPE;
  *blocks = (unsigned)n;
  return EFQAT_OK;
}
static int launch_stage(const XentStageArgs& g, int dtype, hipStream_t st) {
  unsigned blocks;
  if (const int rc = stage_blocks(std::max(g.dst_rows, g.clear ? g.T : 0), g.pitch, &blocks)) return rc;
  if (dtype == EFQAT_F32) EFQAT_TRY(launch((k_xent_stage<float, 3>), dim3(blocks), dim3(256), 0, st, g));
  else EFQAT_TRY(launch((k_xent_stage<bf16_t, 1>), dim3(blocks), dim3(256), 0, st, g));
  return EFQAT_OK;
}

static int check_xent(const void* h, int64_t ldh, const void* w, int64_t ldw, int dtype, int64_t T, int64_t D, int64_t V,
                      const int64_t* targets, int reduction, const void* ws) {
  // token slots and classes are 32-bit numbers, offsets inside a tile of 256 rows too
  if (T <= 0 || D <= 0 || V <= 0 || T > INT64_C(1) << 30 || V > INT64_C(1) << 30 || D > INT64_C(1) << 20 || ldh < D || ldw < D ||
      ldw > INT64_C(1) << 22)
    return EFQAT_ERR_BAD_SHAPE;
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

extern "C" size_t efqat_linear_xent_fwd_workspace_bytes(int64_t T, int64_t D, int64_t V, int dtype) {
  if (T <= 0 || D <= 0 || V <= 0 || !known_dtype(dtype)) return 256;
  return xent_ws(nullptr, xent_plan(T, D, V, dtype, false), T, V, false).bytes;
}
extern "C" size_t efqat_linear_xent_bwd_workspace_bytes(int64_t T, int64_t D, int64_t V, int dtype) {
  if (T <= 0 || D <= 0 || V <= 0 || !known_dtype(dtype)) return 256;
  return xent_ws(nullptr, xent_plan(T, D, V, dtype, true), T, V, true).bytes;
}

extern "C" int efqat_linear_xent_fwd(const void* h, int64_t ldh, const void* w, int64_t ldw, int dtype, int64_t T, int64_t D, int64_t V,
                                     const int64_t* targets, int64_t ignore_index, int reduction, float* loss, float* lse,
                                     int32_t* n_valid, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_xent(h, ldh, w, ldw, dtype, T, D, V, targets, reduction, ws)) return rc;
  if (!loss || !lse) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(loss) || !aligned4(lse) || !aligned4(n_valid)) return EFQAT_ERR_ALIGNMENT;
  const XentPlan p = xent_plan(T, D, V, dtype, false);
  const XentWs k = xent_ws(ws, p, T, V, false);
  if (ws_bytes < k.bytes) return EFQAT_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const bool none = reduction == EFQAT_XENT_NONE;

  XentRowsArgs r = {};
  r.targets = targets; r.T = T; r.V = V; r.ignore = ignore_index;
  r.rows = k.rows; r.target = k.target; r.n_valid = k.n_valid; r.n_out = n_valid;
  r.loss = none ? loss : nullptr; r.lse = lse;
  EFQAT_TRY(launch(k_xent_rows, dim3(1), dim3(1024), 0, st, r));

  XentStageArgs sh = {};
  sh.src = h; sh.ld = ldh; sh.cols = D; sh.pitch = p.Dp; sh.rows = k.rows; sh.n_valid = k.n_valid; sh.dst_rows = p.slots; sh.dst = k.h;
  EFQAT_TRY(launch_stage(sh, dtype, st));

  for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
    const int64_t n = std::min(p.piece, V - v0);
    XentGemmArgs g = {};
    g.segments = p.parts == 3 ? 6 : 1;
    if (p.stage_w) {
      XentStageArgs sw = {};
      sw.src = (const char*)w + v0 * ldw * (dtype == EFQAT_F32 ? 4 : 2);
      sw.ld = ldw; sw.cols = D; sw.pitch = p.Dp; sw.n_rows = n; sw.dst_rows = n; sw.dst = k.w;
      EFQAT_TRY(launch_stage(sw, dtype, st));
      g.A = k.w; g.lda = p.parts * p.Dp;
    } else {
      g.A = (const bf16_t*)w + v0 * ldw; g.lda = ldw;
    }
    g.B = k.h; g.ldb = p.parts * p.Dp;
    g.a_part = g.b_part = (int)p.Dp;
    g.M = (int)n; g.N = (int)T; g.K = (int)p.Dp;
    g.count_n = 1; g.n_valid = k.n_valid;
    g.class0 = (int)v0; g.target = k.target; g.part = k.part; g.target_logit = k.target_logit; g.slots = (int)p.slots;
    EFQAT_TRY(launch_xent_tile<false, false, XG_LSE>(p.bt, g, st));
  }

  // tiles of a piece are whole but for the last piece's: pieces are multiples of 256 classes
  EFQAT_TRY(launch(k_xent_join, dim3((unsigned)ceil_div(T, 64)), dim3(256), 0, st, k.part, (int)ceil_div(V, p.bt), (int)p.slots, k.n_valid,
                     k.rows, k.target_logit, lse, none ? loss : (float*)nullptr, k.slot_loss));
  if (!none) {
    EFQAT_TRY(launch(k_xent_reduce_loss, dim3(1), dim3(1024), 0, st, k.slot_loss, k.n_valid, reduction == EFQAT_XENT_MEAN ? 1 : 0, loss));
  }
  return EFQAT_OK;
}

extern "C" int efqat_linear_xent_bwd(const void* h, int64_t ldh, const void* w, int64_t ldw, int dtype, int64_t T, int64_t D, int64_t V,
                                     const int64_t* targets, int64_t ignore_index, int reduction, const float* lse, const float* dloss,
                                     void* dh, int64_t lddh, void* dw, int64_t lddw, void* ws, size_t ws_bytes, void* stream) {
  if (const int rc = check_xent(h, ldh, w, ldw, dtype, T, D, V, targets, reduction, ws)) return rc;
  if ((dh && lddh < D) || (dw && lddw < D)) return EFQAT_ERR_BAD_SHAPE;
  if (!lse || (!dh && !dw)) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(lse) || !aligned4(dloss) || !aligned_for(dh, dtype) || !aligned_for(dw, dtype)) return EFQAT_ERR_ALIGNMENT;
  const XentPlan p = xent_plan(T, D, V, dtype, true);
  const XentWs k = xent_ws(ws, p, T, V, true);
  if (ws_bytes < k.bytes) return EFQAT_ERR_WORKSPACE;
  hipStream_t st = (hipStream_t)stream;
  const int64_t elem = dtype == EFQAT_F32 ? 4 : 2;

  XentRowsArgs r = {};
  r.targets = targets; r.T = T; r.V = V; r.ignore = ignore_index;
  r.rows = k.rows; r.target = k.target; r.n_valid = k.n_valid;
  r.lse_in = lse; r.dloss = dloss; r.reduction = reduction; r.slot_lse = k.slot_lse; r.slot_scale = k.slot_scale;
  EFQAT_TRY(launch(k_xent_rows, dim3(1), dim3(1024), 0, st, r));

  XentStageArgs sh = {};
  sh.src = h; sh.ld = ldh; sh.cols = D; sh.pitch = p.Dp; sh.rows = k.rows; sh.n_valid = k.n_valid; sh.dst_rows = p.slots; sh.dst = k.h;
  sh.targets = targets; sh.T = T; sh.V = V; sh.ignore = ignore_index; sh.clear = dh; sh.ld_clear = lddh;
  EFQAT_TRY(launch_stage(sh, dtype, st));

  for (int64_t v0 = 0; v0 < V; v0 += p.piece) {
    const int64_t n = std::min(p.piece, V - v0);
    const bool first = v0 == 0, last = v0 + p.piece >= V;
    XentGemmArgs g = {};
    g.segments = p.parts == 3 ? 6 : 1;
    g.n_valid = k.n_valid;
    const bf16_t* W = (const bf16_t*)w + v0 * ldw;
    int64_t ldW = ldw;
    if (p.stage_w) {
      XentStageArgs sw = {};
      sw.src = (const char*)w + v0 * ldw * elem;
      sw.ld = ldw; sw.cols = D; sw.pitch = p.Dp; sw.n_rows = n; sw.dst_rows = round_up(n, 64); sw.dst = k.w;
      EFQAT_TRY(launch_stage(sw, dtype, st));
      W = k.w; ldW = p.parts * p.Dp;
    }
    const int64_t ldG = p.parts * p.piece;
    {
      XentGemmArgs q = g;
      q.A = W; q.lda = ldW; q.a_part = (int)p.Dp;
      q.B = k.h; q.ldb = p.parts * p.Dp; q.b_part = (int)p.Dp;
      q.M = (int)n; q.N = (int)T; q.K = (int)p.Dp; q.count_n = 1;
      q.class0 = (int)v0; q.target = k.target; q.lse = k.slot_lse; q.scale = k.slot_scale; q.grad = k.grad; q.grad_pitch = (int)p.piece;
      EFQAT_TRY(launch_xent_tile<false, false, XG_GRAD>(p.bt, q, st));
    }
    if (dw) {
      XentGemmArgs q = g;
      q.A = k.h; q.lda = p.parts * p.Dp; q.a_part = (int)p.Dp; q.a_cols = (int)p.Dp;
      q.B = k.grad; q.ldb = ldG; q.b_part = (int)p.piece; q.b_cols = (int)p.piece;
      q.M = (int)D; q.N = (int)n; q.K = (int)T; q.count_k = 1;
      q.split_blocks = p.blocks_dw; q.acc = k.acc_dw;
      q.out = (char*)dw + v0 * lddw * elem; q.out_dtype = dtype; q.ldo = lddw;
      EFQAT_TRY(launch_xent_tile<true, true, XG_OUT>(p.bt_dw, q, st));
      q.tiles_m = (int)ceil_div(D, p.bt_dw);
      if (xent_split((int)(q.tiles_m * ceil_div(n, p.bt_dw)), (int)ceil_div(T, 64), p.blocks_dw) > 1) {   // for enough tokens
        if (dtype == EFQAT_F32) EFQAT_TRY(launch(k_xent_join_slices<float>, dim3(1024), dim3(256), 0, st, q, p.bt_dw));
        else EFQAT_TRY(launch(k_xent_join_slices<bf16_t>, dim3(1024), dim3(256), 0, st, q, p.bt_dw));
      }
    }
    if (dh) {
      XentGemmArgs q = g;
      q.A = W; q.lda = ldW; q.a_part = (int)p.Dp; q.a_cols = (int)p.Dp; q.a_rows = p.stage_w ? 0 : (int)n;
      q.B = k.grad; q.ldb = ldG; q.b_part = (int)p.piece;
      q.M = (int)D; q.N = (int)T; q.K = (int)n; q.count_n = 1;
      q.split_blocks = p.blocks_dh; q.split_stages = (int)ceil_div(std::min(p.piece, V), 64);
      q.acc = k.acc_dh; q.acc_add = first ? 0 : 1; q.acc_write = last ? 0 : 1;
      q.out = dh; q.out_dtype = dtype; q.ldo = lddh; q.rows = k.rows;
      EFQAT_TRY(launch_xent_tile<true, false, XG_OUT>(p.bt_dh, q, st));
      q.tiles_m = (int)ceil_div(D, p.bt_dh);
      if (last && xent_split(q.tiles_m, q.split_stages, q.split_blocks) > 1) {   // for few enough tokens
        if (dtype == EFQAT_F32) EFQAT_TRY(launch(k_xent_join_slices<float>, dim3(1024), dim3(256), 0, st, q, p.bt_dh));
        else EFQAT_TRY(launch(k_xent_join_slices<bf16_t>, dim3(1024), dim3(256), 0, st, q, p.bt_dh));
      }
    }
  }
  return EFQAT_OK;
}
