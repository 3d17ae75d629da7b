// Layer norm over the columns of [rows][cols], forward and backward.
//
//   forward   xhat = (x - mean) rstd,  rstd = 1 / sqrt(var + eps),  y = xhat w + b
//   backward  g = dy w,  dx = rstd (g - mean_j g - xhat mean_j (g xhat)),  dw = sum_rows dy xhat,  db = sum_rows dy
//
// Bound by HBM: a row is read once into registers (TPR lanes, NIT chunks of 8 columns each), its sums are taken there - the
// variance from the differences to the mean, so that an offset of the row costs no digits - and its outputs leave from there.
// A block keeps its columns' parameters and, backward, their sums over all its rows in registers; the rows that come next are
// requested before the present ones are worked on.  The sums of the blocks are added in a second pass, in a fixed order.
// Rows longer than the registers hold (kNormMaxCols, kNormBwdMaxCols), and shorter than a chunk, are read again for every step.
//
// bf16, one call after another on the same buffers (which the last-level cache holds).  8192 x 4096: forward 22.6 us (134 MB, 5.9 TB/s),
// input kept 28.4, backward 38.1 (201 MB, 5.3 TB/s), from the checkpoint 34.2.  12288 x 768: 9.6, 12.4, 16.8 (57 MB, 3.4 TB/s) and 17.0 us:
// narrow rows are bound by the instructions a value takes (two sums, the code) and by the way through a row, load to store, that a block
// walks a few times; 4 us of the backward are the second pass, mostly its launch.  1 x 4096: 2.5 us of kernel in 6.4 us a call.
#include "rows.hpp"

#include <algorithm>

namespace efqat {

constexpr int64_t kNormMaxCols = 16384, kNormBwdMaxCols = 8192;
constexpr int kNormLongCols = 2048;                   // columns of a block of the second long-row kernel

__device__ __forceinline__ int chunk_len(int64_t cols, int64_t col) {
  const int64_t left = cols - col;
  return left > 8 ? 8 : (int)(left < 0 ? 0 : left);
}

// Sums of two values over the TPR lanes of a row; every lane of the block calls it.  The buffers alternate, so that one
// barrier a call is enough.
template <int THREADS, int TPR>
struct RowSum {
  static constexpr int WPR = TPR / 64, WAVES = THREADS / 64;
  float2 (*buf)[WAVES];
  int turn = 0;
  __device__ __forceinline__ float operator()(float a) { return (*this)(a, 0.0f).x; }
  __device__ __forceinline__ float2 operator()(float a, float b) {
    a = wave_total(a);
    b = wave_total(b);
    if constexpr (WPR == 1) return make_float2(a, b);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) buf[turn][wave] = make_float2(a, b);
    __syncthreads();
    float2 s = make_float2(0.0f, 0.0f);
    const int w0 = wave / WPR * WPR;
#pragma unroll
    for (int i = 0; i < WPR; ++i) {
      const float2 o = buf[turn][w0 + i];
      s.x += o.x;
      s.y += o.y;
    }
    turn ^= 1;
    return s;
  }
};

// From the sums of d = x - mean and of d^2: what the mean has lost to rounding is put back (the sum of d is not quite zero), and what
// that adds to the squares taken off.  A row with a NaN or an infinity has the mean that its sum says and a NaN for rstd; one whose
// squares alone leave fp32 has rstd 0 (the product of the second step is not rounded before it is taken off an infinite sum).
__device__ __forceinline__ float norm_rstd(float2 sums, float inv_cols, float eps, float* mean) {
  const float more = sums.x * inv_cols, var = fmaf(-more, more, sums.y * inv_cols);
  *mean += fabsf(more) < INFINITY ? more : 0.0f;
  return 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);
}

struct NormFwdArgs {
  const void* x;
  const float *w, *b;
  void* y;
  float *mean, *rstd;
  int8_t* codes;
  float* scales;
  int64_t rows, cols, ldx, ldy;
  float eps;
};

__device__ __forceinline__ void load_param(const float* p, float dflt, int64_t col, int n, float (&v)[8]) {
  if (p) {
    load_chunk(p + col, n).get(v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = dflt;
  }
}

// the same for rows that are read without a branch
__device__ __forceinline__ void load_param(const float* p, float dflt, const ChunkPlace& at, float (&v)[8]) {
  if (p) {
    Raw8<float> r;
    r.load(p + at.at);
    get_chunk(r, at, v);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = dflt;
  }
}

template <typename T, int THREADS, int TPR, int NIT, bool KEEP>
__global__ __launch_bounds__(THREADS) void k_norm_fwd(const NormFwdArgs g) {
  constexpr int RPB = THREADS / TPR;
  __shared__ float2 sums[2][THREADS / 64];
  RowSum<THREADS, TPR> row_sum{sums};
  const int t = threadIdx.x % TPR;
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);             // rows are whole wavefronts': their addresses are scalar
  ChunkPlace at[NIT];
  float w[NIT][8], b[NIT][8];
#pragma unroll
  for (int i = 0; i < NIT; ++i) at[i] = ChunkPlace(g.cols, (i * TPR + t) * 8);
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  const float inv_cols = 1.0f / (float)g.cols;
  Raw8<T> next[NIT];
  auto request = [&](int64_t r) {
#pragma unroll
    for (int i = 0; i < NIT; ++i) next[i].load((const T*)g.x + (r < g.rows ? r : g.rows - 1) * g.ldx + at[i].at);
  };
  request(row);
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    load_param(g.w, 1.0f, at[i], w[i]);
    load_param(g.b, 0.0f, at[i], b[i]);
  }
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < g.rows; base += step, row += step) {
    float v[NIT][8];
#pragma unroll
    for (int i = 0; i < NIT; ++i) get_chunk(next[i], at[i], v[i]);
    request(row + step);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[i][j];
    float mean = row_sum(s) * inv_cols, q = 0.0f, rest = 0.0f;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
      if (at[i].n == 8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = v[i][j] - mean;
          rest += d;
          q = fmaf(d, d, q);
        }
      } else if (at[i].n > 0) {
#pragma unroll
        for (int j = 0; j < 7; ++j) {
          const float d = j < at[i].n ? v[i][j] - mean : 0.0f;
          rest += d;
          q = fmaf(d, d, q);
        }
      }
    }
    const float rstd = norm_rstd(row_sum(rest, q), inv_cols, g.eps, &mean);
    if (row >= g.rows) continue;                      // the whole wavefront: its lanes are of one row
    if (t == 0) {
      if (g.mean) g.mean[row] = mean;
      if (g.rstd) g.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = fmaf((v[i][j] - mean) * rstd, w[i][j], b[i][j]);
      const int col = (i * TPR + t) * 8;
      store_chunk((T*)g.y + row * g.ldy + col, at[i].n, o);
      if constexpr (KEEP) {
        float scale;
        const uint2 c = ckpt_encode(v[i], &scale);
        if (col < ckpt_pitch(g.cols)) *reinterpret_cast<uint2*>(g.codes + row * ckpt_pitch(g.cols) + col) = c;
        if ((t & (kGroupLanes - 1)) == 0 && col < g.cols) g.scales[row * ckpt_groups(g.cols) + col / kCkptGroup] = scale;
      }
    }
  }
}

// rows beyond the registers: one block a row, which it reads three times (from the caches after the first)
template <typename T, bool KEEP>
__global__ __launch_bounds__(1024) void k_norm_fwd_long(const NormFwdArgs g) {
  __shared__ float2 sums[2][16];
  RowSum<1024, 1024> row_sum{sums};
  const float inv_cols = 1.0f / (float)g.cols;
  const int64_t whole = round_up(g.cols, kCkptGroup);                // groups are whole: all their lanes take part
  for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
    const T* x = (const T*)g.x + row * g.ldx;
    float s = 0.0f, q = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < g.cols; c += 8192) {
      float v[8];
      load_chunk(x + c, chunk_len(g.cols, c)).get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) s += v[j];
    }
    float mean = row_sum(s) * inv_cols, rest = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < g.cols; c += 8192) {
      const int n = chunk_len(g.cols, c);
      float v[8];
      load_chunk(x + c, n).get(v);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = j < n ? v[j] - mean : 0.0f;
        rest += d;
        q = fmaf(d, d, q);
      }
    }
    const float rstd = norm_rstd(row_sum(rest, q), inv_cols, g.eps, &mean);
    if (threadIdx.x == 0) {
      if (g.mean) g.mean[row] = mean;
      if (g.rstd) g.rstd[row] = rstd;
    }
    for (int64_t c = threadIdx.x * 8; c < whole; c += 8192) {
      const int n = chunk_len(g.cols, c);
      float v[8], w[8], b[8];
      load_chunk(x + c, n).get(v);
      load_param(g.w, 1.0f, c, n, w);
      load_param(g.b, 0.0f, c, n, b);
      if constexpr (KEEP) {
        float scale;
        const uint2 k = ckpt_encode(v, &scale);
        if (c < ckpt_pitch(g.cols)) *reinterpret_cast<uint2*>(g.codes + row * ckpt_pitch(g.cols) + c) = k;
        if ((threadIdx.x & (kGroupLanes - 1)) == 0) g.scales[row * ckpt_groups(g.cols) + c / kCkptGroup] = scale;
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] = fmaf((v[j] - mean) * rstd, w[j], b[j]);
      store_chunk((T*)g.y + row * g.ldy + c, n, v);
    }
  }
}

struct NormBwdArgs {
  const void *dy, *x;                                 // x or codes and scales
  const int8_t* codes;
  const float* scales;
  const float *mean, *rstd, *w;
  void* dx;
  float* part;                                        // [blocks][2][cols]: sums of dy xhat, of dy; one block: unused
  float *dw, *db;                                     // nullable
  float2* row_sums;                                   // long rows: means of g and of g xhat
  int64_t rows, cols, lddy, ldx, lddx;
};

// a chunk of the input of the forward, from itself or from its checkpoint
template <typename T, bool CKPT>
struct InputChunk {
  Raw8<T> raw;
  uint2 q;
  float scale;
  __device__ __forceinline__ void request(const NormBwdArgs& g, int64_t row, int64_t col, int n) {
    if constexpr (CKPT) {
      q = make_uint2(0, 0);
      scale = 0.0f;
      if (n > 0) {
        q = *reinterpret_cast<const uint2*>(g.codes + row * ckpt_pitch(g.cols) + col);
        scale = g.scales[row * ckpt_groups(g.cols) + col / kCkptGroup];
      }
    } else {
      raw = load_chunk((const T*)g.x + row * g.ldx + col, n);
    }
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
    if constexpr (CKPT) ckpt_decode(q, scale, v);
    else raw.get(v);
  }
  // without a branch, in rows of 8 columns and more (codes behind the columns are zeros)
  __device__ __forceinline__ void request(const NormBwdArgs& g, int64_t row, int64_t col, const ChunkPlace& at) {
    if constexpr (CKPT) {
      const int64_t pitch = ckpt_pitch(g.cols), groups = ckpt_groups(g.cols);
      q = *reinterpret_cast<const uint2*>(g.codes + row * pitch + (col < pitch ? col : pitch - 8));
      scale = g.scales[row * groups + (col < g.cols ? col / kCkptGroup : groups - 1)];
    } else {
      raw.load((const T*)g.x + row * g.ldx + at.at);
    }
  }
  __device__ __forceinline__ void get(const ChunkPlace& at, float (&v)[8]) const {
    if constexpr (CKPT) ckpt_decode(q, scale, v);
    else get_chunk(raw, at, v);
  }
};

template <typename T, bool CKPT, int THREADS, int TPR, int NIT>
__global__ __launch_bounds__(THREADS, 4) void k_norm_bwd(const NormBwdArgs g) {
  constexpr int RPB = THREADS / TPR;
  __shared__ float2 sums[2][THREADS / 64];
  __shared__ float red[RPB > 1 ? THREADS * 16 : 1];
  RowSum<THREADS, TPR> row_sum{sums};
  const int t = threadIdx.x % TPR;
  const int sub = __builtin_amdgcn_readfirstlane(threadIdx.x / TPR);             // rows are whole wavefronts': their addresses are scalar
  ChunkPlace at[NIT];
  float w[NIT][8], aw[NIT][8], ab[NIT][8];
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    at[i] = ChunkPlace(g.cols, (i * TPR + t) * 8);
#pragma unroll
    for (int j = 0; j < 8; ++j) aw[i][j] = ab[i][j] = 0.0f;
  }
  const int64_t step = (int64_t)gridDim.x * RPB;
  int64_t row = (int64_t)blockIdx.x * RPB + sub;
  const float inv_cols = 1.0f / (float)g.cols;
  Raw8<T> next_dy[NIT];
  InputChunk<T, CKPT> next_x[NIT];
  float next_mean = 0.0f, next_rstd = 0.0f;
  auto request = [&](int64_t r) {
    r = r < g.rows ? r : g.rows - 1;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
      next_dy[i].load((const T*)g.dy + r * g.lddy + at[i].at);
      next_x[i].request(g, r, (i * TPR + t) * 8, at[i]);
    }
    next_mean = g.mean[r];
    next_rstd = g.rstd[r];
  };
  request(row);
#pragma unroll
  for (int i = 0; i < NIT; ++i) load_param(g.w, 1.0f, at[i], w[i]);
  for (int64_t base = (int64_t)blockIdx.x * RPB; base < g.rows; base += step, row += step) {
    float d[NIT][8], xh[NIT][8];
    const bool in = row < g.rows;
    const float mean = in ? next_mean : 0.0f, rstd = in ? next_rstd : 0.0f;
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
      get_chunk(next_dy[i], at[i], d[i]);
      next_x[i].get(at[i], xh[i]);
    }
    request(row + step);
    if (!in) {                                        // nothing of a row that does not exist is summed
#pragma unroll
      for (int i = 0; i < NIT; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) d[i][j] = xh[i][j] = 0.0f;
    }
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int i = 0; i < NIT; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[i][j] = (xh[i][j] - mean) * rstd;
        aw[i][j] = fmaf(d[i][j], xh[i][j], aw[i][j]);
        ab[i][j] += d[i][j];
        d[i][j] *= w[i][j];
        s1 += d[i][j];
        s2 = fmaf(d[i][j], xh[i][j], s2);
      }
    const float2 s = row_sum(s1, s2);
    const float m1 = s.x * inv_cols, m2 = s.y * inv_cols;
    if (!in) continue;                                // the whole wavefront: its lanes are of one row
#pragma unroll
    for (int i = 0; i < NIT; ++i) {
#pragma unroll
      for (int j = 0; j < 8; ++j) d[i][j] = (d[i][j] - m1 - xh[i][j] * m2) * rstd;
      store_chunk((T*)g.dx + row * g.lddx + (i * TPR + t) * 8, at[i].n, d[i]);
    }
  }
  if (!g.dw && !g.db) return;
  // one block: the sums are the gradients
  float* ow = gridDim.x == 1 ? g.dw : g.part + (int64_t)blockIdx.x * 2 * g.cols;
  float* ob = gridDim.x == 1 ? g.db : ow + g.cols;
#pragma unroll
  for (int i = 0; i < NIT; ++i) {
    if constexpr (RPB > 1) {
      // the rows of the block that ran beside each other, in their order
      __syncthreads();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        red[j * THREADS + threadIdx.x] = aw[i][j];
        red[(8 + j) * THREADS + threadIdx.x] = ab[i][j];
      }
      __syncthreads();
      if (sub == 0) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float a = 0.0f, b = 0.0f;
#pragma unroll
          for (int r = 0; r < RPB; ++r) {
            a += red[j * THREADS + r * TPR + t];
            b += red[(8 + j) * THREADS + r * TPR + t];
          }
          aw[i][j] = a;
          ab[i][j] = b;
        }
      }
    }
    if (sub == 0) {
      if (ow) store_chunk(ow + (i * TPR + t) * 8, at[i].n, aw[i]);
      if (ob) store_chunk(ob + (i * TPR + t) * 8, at[i].n, ab[i]);
    }
  }
}

// Long rows, first pass: the two means of a row.  Two readings of the rows and three launches: 2048 x 12288 bf16 41.0 us (floor of the bytes,
// read once, 29), 16 / 64 / 128 rows 13.8 / 14.3 / 16.0 us, where the second pass has 12 to 96 blocks and each walks its eight rows.
template <typename T, bool CKPT>
__global__ __launch_bounds__(1024) void k_norm_bwd_long_rows(const NormBwdArgs g) {
  __shared__ float2 sums[2][16];
  RowSum<1024, 1024> row_sum{sums};
  const float inv_cols = 1.0f / (float)g.cols;
  for (int64_t row = blockIdx.x; row < g.rows; row += gridDim.x) {
    const float mean = g.mean[row], rstd = g.rstd[row];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t c = threadIdx.x * 8; c < g.cols; c += 8192) {
      const int n = chunk_len(g.cols, c);
      InputChunk<T, CKPT> in;
      float d[8], x[8], w[8];
      in.request(g, row, c, n);
      load_chunk((const T*)g.dy + row * g.lddy + c, n).get(d);
      load_param(g.w, 1.0f, c, n, w);
      in.get(x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float gj = d[j] * w[j];
        s1 += gj;
        s2 = fmaf(gj, (x[j] - mean) * rstd, s2);
      }
    }
    const float2 s = row_sum(s1, s2);
    if (threadIdx.x == 0) g.row_sums[row] = make_float2(s.x * inv_cols, s.y * inv_cols);
  }
}
// Second pass: dX, and the sums over the rows of a block's columns.
template <typename T, bool CKPT>
__global__ __launch_bounds__(256) void k_norm_bwd_long_cols(const NormBwdArgs g) {
  const int64_t c = (int64_t)blockIdx.x * kNormLongCols + threadIdx.x * 8;
  const int n = chunk_len(g.cols, c);
  if (n <= 0) return;
  float w[8], aw[8], ab[8];
  load_param(g.w, 1.0f, c, n, w);
#pragma unroll
  for (int j = 0; j < 8; ++j) aw[j] = ab[j] = 0.0f;
  constexpr int NR = 4;                               // rows whose loads are in flight together
  for (int64_t r0 = blockIdx.y; r0 < g.rows; r0 += NR * (int64_t)gridDim.y) {
    InputChunk<T, CKPT> in[NR];
    Raw8<T> dy[NR];
    float mean[NR], rstd[NR];
    float2 m[NR];
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int64_t next = r0 + u * (int64_t)gridDim.y, row = next < g.rows ? next : r0;
      in[u].request(g, row, c, n);
      dy[u] = load_chunk((const T*)g.dy + row * g.lddy + c, n);
      mean[u] = g.mean[row];
      rstd[u] = g.rstd[row];
      m[u] = g.row_sums[row];
    }
#pragma unroll
    for (int u = 0; u < NR; ++u) {
      const int64_t row = r0 + u * (int64_t)gridDim.y;
      if (row >= g.rows) break;
      float d[8], x[8];
      dy[u].get(d);
      in[u].get(x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float xh = (x[j] - mean[u]) * rstd[u];
        aw[j] = fmaf(d[j], xh, aw[j]);
        ab[j] += d[j];
        d[j] = (d[j] * w[j] - m[u].x - xh * m[u].y) * rstd[u];
      }
      store_chunk((T*)g.dx + row * g.lddx + c, n, d);
    }
  }
  if (!g.dw && !g.db) return;
  float* ow = gridDim.y == 1 ? g.dw : g.part + (int64_t)blockIdx.y * 2 * g.cols;
  float* ob = gridDim.y == 1 ? g.db : ow + g.cols;
  if (ow) store_chunk(ow + c, n, aw);
  if (ob) store_chunk(ob + c, n, ab);
}

// The blocks' sums, 32 columns a block (of the 2 cols that dw and db have together), dealt to 32 groups of lanes whose sums are added in
// double precision in a fixed order.
__global__ __launch_bounds__(1024) void k_norm_finish(const float* __restrict__ part, int nblk, int64_t cols, float* __restrict__ dw,
                                                      float* __restrict__ db) {
  __shared__ double red[32][33];
  const int lane = threadIdx.x & 31, grp = threadIdx.x >> 5;
  const int64_t c = (int64_t)blockIdx.x * 32 + lane;
  double s = 0.0;
  if (c < 2 * cols) {
    for (int i = grp; i < nblk; i += 512) {           // sixteen independent loads in flight
      float v[16];
#pragma unroll
      for (int u = 0; u < 16; ++u) v[u] = part[(int64_t)(i + 32 * u < nblk ? i + 32 * u : nblk - 1) * 2 * cols + c];
#pragma unroll
      for (int u = 0; u < 16; ++u) s += i + 32 * u < nblk ? (double)v[u] : 0.0;
    }
  }
  red[grp][lane] = s;
  __syncthreads();
  // 32 lanes take a column each: the groups of a column pairwise, by the lanes of half a wavefront
  double t = red[lane][grp];                          // column grp, group lane
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) t += __shfl_xor(t, o, 32);
  const int64_t k = (int64_t)blockIdx.x * 32 + grp;
  if (lane == 0 && k < 2 * cols) {
    float* out = k < cols ? dw : db;
    if (out) out[k < cols ? k : k - cols] = (float)t;
  }
}

// most blocks: `most`; every block walks as many rows as the others, or one step fewer
static unsigned even_blocks(int64_t rows, int64_t rows_per_block, int64_t most) {
  const int64_t steps = ceil_div(ceil_div(rows, rows_per_block), most);
  return (unsigned)ceil_div(rows, rows_per_block * steps);
}

// Blocks of the backward pass: as many as the chip holds (two of 512 threads a CU, one of 1024; a block walks rows, and its sums over
// them are one partial result), fewer where there are fewer rows than that.
static int64_t norm_rows_per_block(int64_t cols) { return cols <= 512 ? 8 : cols <= 1024 ? 4 : cols <= 2048 ? 2 : 1; }
static bool norm_bwd_long(int64_t cols) { return cols < 8 || cols > kNormBwdMaxCols; }
static int64_t norm_bwd_blocks(int64_t rows, int64_t cols) {
  // long rows: blocks of 2048 columns, 1024 in all; eight rows a block at least, whose sums cost a quarter of what the rows do
  if (norm_bwd_long(cols)) return std::min<int64_t>(ceil_div(rows, 8), std::max<int64_t>(1, 1024 / ceil_div(cols, kNormLongCols)));
  return even_blocks(rows, norm_rows_per_block(cols), cols <= 4096 ? 512 : 256);
}

// A row by TPR lanes of one chunk (NIT = 1) or two.  One chunk a lane is the shorter way of one row, two keep more bytes in flight and
// need half of the wavefronts to talk to each other: one where the chip holds all rows' blocks at once (2048 threads a CU), else two in
// blocks that walk the rows, all as many.  One against two, us: 16 x 768 bf16 3.22 / 3.63, 2049 x 777 4.59 / 4.92, 12288 x 768 11.7 /
// 10.9, 8192 x 4096 23.0 / 22.1, 2048 x 8192 16.0 / 13.1 (buffers that the last-level cache holds).  Blocks that walk: 1024 threads a CU;
// with 2048 12288 x 768 takes 9.4 instead of 9.5, 8192 x 4096 fp32 with its checkpoint 60 instead of 55, 2048 x 8192 14.8 instead of 13.4.
template <typename T, bool KEEP>
static int launch_norm_fwd(const NormFwdArgs& g, hipStream_t st) {
  const int64_t cols = g.cols;
  if (cols < 8 || cols > kNormMaxCols) return launch((k_norm_fwd_long<T, KEEP>), dim3((unsigned)std::min<int64_t>(g.rows, 512)), dim3(1024), 0, st, g);
#define EFQAT_NORM(THREADS, TPR, NIT) \
  return launch((k_norm_fwd<T, THREADS, TPR, NIT, KEEP>), dim3(even_blocks(g.rows, (THREADS) / (TPR), 256 * (NIT == 1 ? 2048 : 1024) / (THREADS))), dim3(THREADS), 0, st, g)
  auto at_once = [&](int threads, int tpr) { return ceil_div(g.rows, threads / tpr) <= 256 * 2048 / threads; };
  if (cols <= 512) EFQAT_NORM(256, 64, 1);
  if (cols <= 1024) { if (at_once(256, 128)) EFQAT_NORM(256, 128, 1); EFQAT_NORM(256, 64, 2); }
  if (cols <= 2048) { if (at_once(256, 256)) EFQAT_NORM(256, 256, 1); EFQAT_NORM(256, 128, 2); }
  if (cols <= 4096) { if (at_once(512, 512)) EFQAT_NORM(512, 512, 1); EFQAT_NORM(256, 256, 2); }
  if (cols <= 8192) { if (at_once(1024, 1024)) EFQAT_NORM(1024, 1024, 1); EFQAT_NORM(512, 512, 2); }
  EFQAT_NORM(1024, 1024, 2);
#undef EFQAT_NORM
}

template <typename T, bool CKPT>
static int launch_norm_bwd(const NormBwdArgs& g, int64_t blocks, hipStream_t st) {
  const int64_t cols = g.cols;
  if (norm_bwd_long(cols)) {
    EFQAT_TRY(launch((k_norm_bwd_long_rows<T, CKPT>), dim3((unsigned)std::min<int64_t>(g.rows, 512)), dim3(1024), 0, st, g));
    return launch((k_norm_bwd_long_cols<T, CKPT>), dim3((unsigned)ceil_div(cols, kNormLongCols), (unsigned)blocks), dim3(256), 0, st, g);
  }
#define EFQAT_NORM(THREADS, TPR) return launch((k_norm_bwd<T, CKPT, THREADS, TPR, 1>), dim3((unsigned)blocks), dim3(THREADS), 0, st, g)
  if (cols <= 512) EFQAT_NORM(512, 64);
  if (cols <= 1024) EFQAT_NORM(512, 128);
  if (cols <= 2048) EFQAT_NORM(512, 256);
  if (cols <= 4096) EFQAT_NORM(512, 512);
  EFQAT_NORM(1024, 1024);
#undef EFQAT_NORM
}

}  // namespace efqat

using namespace efqat;

extern "C" int efqat_layer_norm_fwd(const void* x, int64_t ldx, int dtype, int64_t rows, int64_t cols, const float* weight,
                                    const float* bias, float eps, void* y, int64_t ldy, float* mean, float* rstd, int8_t* x_codes,
                                    float* x_scales, void* stream) {
  if (rows <= 0 || cols <= 0 || cols > INT32_MAX || ldx < cols || ldy < cols || !(eps >= 0.0f)) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  const bool keep = x_codes != nullptr || x_scales != nullptr;
  if (!x || !y || (keep && (!x_codes || !x_scales))) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(x, dtype) || !aligned_for(y, dtype) || !aligned4(weight) || !aligned4(bias) || !aligned4(mean) || !aligned4(rstd) ||
      !aligned16(x_codes) || !aligned4(x_scales))
    return EFQAT_ERR_ALIGNMENT;
  const NormFwdArgs g = {x, weight, bias, y, mean, rstd, x_codes, x_scales, rows, cols, ldx, ldy, eps};
  hipStream_t st = (hipStream_t)stream;
  EFQAT_TRY(dtype == EFQAT_F32 ? (keep ? launch_norm_fwd<float, true>(g, st) : launch_norm_fwd<float, false>(g, st))
                              : (keep ? launch_norm_fwd<bf16_t, true>(g, st) : launch_norm_fwd<bf16_t, false>(g, st)));
  return EFQAT_OK;
}

extern "C" size_t efqat_layer_norm_bwd_workspace_bytes(int64_t rows, int64_t cols) {
  if (rows <= 0 || cols <= 0 || cols > INT32_MAX) return 256;
  const int64_t blocks = norm_bwd_blocks(rows, cols);
  size_t need = blocks > 1 ? (size_t)round_up(blocks * 2 * cols * (int64_t)sizeof(float), 256) : 0;
  if (norm_bwd_long(cols)) need += (size_t)round_up(rows * (int64_t)sizeof(float2), 256);
  return std::max<size_t>(need, 256);
}

extern "C" int efqat_layer_norm_bwd(const void* dy, int64_t lddy, int dtype, const void* x, int64_t ldx, const int8_t* x_codes,
                                    const float* x_scales, const float* mean, const float* rstd, const float* weight, int64_t rows,
                                    int64_t cols, void* dx, int64_t lddx, float* dweight, float* dbias, void* ws, size_t ws_bytes,
                                    void* stream) {
  const bool ckpt = x == nullptr;
  if (rows <= 0 || cols <= 0 || cols > INT32_MAX || lddy < cols || lddx < cols || (!ckpt && ldx < cols)) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (!dy || !mean || !rstd || !dx || !ws || (ckpt && (!x_codes || !x_scales))) return EFQAT_ERR_NULL_PTR;
  if (ws_bytes < efqat_layer_norm_bwd_workspace_bytes(rows, cols)) return EFQAT_ERR_WORKSPACE;
  if (!aligned_for(dy, dtype) || !aligned_for(x, dtype) || !aligned_for(dx, dtype) || !aligned16(x_codes) || !aligned4(x_scales) ||
      !aligned4(mean) || !aligned4(rstd) || !aligned4(weight) || !aligned4(dweight) || !aligned4(dbias) || ((uintptr_t)ws % 256) != 0)
    return EFQAT_ERR_ALIGNMENT;
  const int64_t blocks = norm_bwd_blocks(rows, cols);
  WsCarver carve(ws);
  float* part = blocks > 1 ? (float*)carve.take((size_t)(blocks * 2 * cols) * sizeof(float)) : nullptr;
  float2* row_sums = norm_bwd_long(cols) ? (float2*)carve.take((size_t)rows * sizeof(float2)) : nullptr;
  const NormBwdArgs g = {dy, x, x_codes, x_scales, mean, rstd, weight, dx, part, dweight, dbias, row_sums, rows, cols, lddy, ldx, lddx};
  hipStream_t st = (hipStream_t)stream;
  EFQAT_TRY(dtype == EFQAT_F32 ? (ckpt ? launch_norm_bwd<float, true>(g, blocks, st) : launch_norm_bwd<float, false>(g, blocks, st))
                              : (ckpt ? launch_norm_bwd<bf16_t, true>(g, blocks, st) : launch_norm_bwd<bf16_t, false>(g, blocks, st)));
  if (blocks > 1 && (dweight || dbias)) {
    EFQAT_TRY(launch(k_norm_finish, dim3((unsigned)ceil_div(2 * cols, 32)), dim3(1024), 0, st, part, (int)blocks, cols, dweight, dbias));
  }
  return EFQAT_OK;
}
