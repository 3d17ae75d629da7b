// Norms of queries and keys for each head with the position rotation in the same pass, forward and backward.
//
//   r = 1 / sqrt(mean_d x_d^2 + eps),  xhat = x r,  n = xhat w
//   y_a = n_a cos t - n_b sin t,  y_b = n_b cos t + n_a sin t  for the F pairs (a, b) of a head,  t = pos[axis(j)] f_j;  y = n behind them
//   dn = the rotation back of dy,  g = dn w,  dx = r (g - xhat mean_d (g xhat)),  dw_d = sum over tokens and heads of dn_d xhat_d
//
// Bound by HBM: what is read is written once.  A lane owns two chunks of 8 features that hold both members of their pairs, so that the
// rotation stays in the lane and the norm is a sum over the D / 16 lanes of a head.  A wavefront takes a token: it makes the F angles
// once (the product in 64 bits, its whole turns taken off, so that far positions keep their place in the circle) and walks the heads.
#include "rows.hpp"

namespace efqat {

struct RopeTensor {
  const void *x, *dy;                                // dy: backward
  void* out;                                         // y, or dx
  int64_t ldx, lddy, ldo;
  const float* w;
  int heads;
};
struct RopeArgs {
  RopeTensor t[2];                                   // queries, keys
  int64_t rows;
  int dim, freqs, axes, norm, slices;
  const int32_t* pos;                                // [axes][rows]
  const int32_t* axis;
  const float* inv_freq;
  float eps;
  float* part;                                       // backward: [blocks][2][dim] sums of dn xhat
};

// cosine and sine of position * f: the turns are formed in 64 bits, their fraction is exact to 2^-25
__device__ __forceinline__ float2 turn_of(const RopeArgs& a, int64_t row, int j) {
  int ax = a.axis ? a.axis[j] : 0;
  ax = ax < 0 ? 0 : ax >= a.axes ? a.axes - 1 : ax;
  const double turns = (double)a.pos[ax * a.rows + row] * (double)a.inv_freq[j] * 0.15915494309189533577;
  float2 cs;
  sincospif((float)(2.0 * (turns - rint(turns))), &cs.y, &cs.x);
  return cs;
}

constexpr int kRopeMostDim = 256;

// Two chunks of a lane: first columns, elements that exist, and the pair of its first element (both are turned with `turn[pair ..]`)
struct RopeLane {
  int col[2], n[2], pair, group;                     // group: head of the pass
  bool turned;
};
template <bool NEXT>
__device__ __forceinline__ RopeLane rope_lane(const RopeArgs& a, int lanes) {
  const int lane = threadIdx.x & 63, c = lane & (lanes - 1);
  RopeLane l;
  l.group = lane / lanes;
  if (!NEXT && 8 * c < a.freqs) {
    l.col[0] = 8 * c;
    l.col[1] = a.freqs + 8 * c;
    l.turned = true;
  } else {
    l.col[0] = NEXT ? 16 * c : 2 * a.freqs + 16 * (c - a.freqs / 8);
    l.col[1] = l.col[0] + 8;
    l.turned = NEXT;
  }
  l.pair = 8 * c;
#pragma unroll
  for (int i = 0; i < 2; ++i) l.n[i] = a.dim - l.col[i] >= 8 ? 8 : 0;
  return l;
}
// rotation (sign 1) or rotation back (-1) of a lane's 16 elements; what has no pair stays as it is, whatever lies beside it
template <bool NEXT>
__device__ __forceinline__ void rope_turn(const RopeLane& l, int freqs, float (&v)[2][8], const float (&cs)[8], const float (&sn)[8], float sign) {
  if constexpr (NEXT) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float x = v[i][2 * j], y = v[i][2 * j + 1], c = cs[4 * i + j], s = sign * sn[4 * i + j];
        const bool in = l.pair + 4 * i + j < freqs;
        v[i][2 * j] = in ? x * c - y * s : x;
        v[i][2 * j + 1] = in ? y * c + x * s : y;
      }
  } else if (l.turned) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = v[0][j], y = v[1][j], s = sign * sn[j];
      v[0][j] = x * cs[j] - y * s;
      v[1][j] = y * cs[j] + x * s;
    }
  }
}
// sum over the lanes of a head
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

template <typename T, bool NEXT, bool BWD>
__global__ __launch_bounds__(256) void k_rope(RopeArgs a, int lanes) {
  __shared__ float2 s_turn[4][kRopeMostDim / 2];
  __shared__ float s_sum[BWD ? 4 : 1][2][BWD ? kRopeMostDim : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RopeLane l = rope_lane<NEXT>(a, lanes);
  const int per_pass = 64 / lanes, pq = (a.t[0].heads + per_pass - 1) / per_pass, pk = (a.t[1].heads + per_pass - 1) / per_pass;
  const int64_t items = a.rows * a.slices;
  float sum[2][2][8] = {};
  for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < items; item += (int64_t)gridDim.x * 4) {
    const int64_t row = item / a.slices;
    const int slice = (int)(item - row * a.slices);
    float cs[8], sn[8];
    if (a.freqs > 0) {
      for (int j = lane; j < a.freqs; j += 64) s_turn[wave][j] = turn_of(a, row, j);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const bool in = l.turned && l.pair + j < a.freqs;
        const float2 t = in ? s_turn[wave][l.pair + j] : make_float2(1.0f, 0.0f);
        cs[j] = t.x;
        sn[j] = t.y;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
    const int first = (pq + pk) * slice / a.slices, last = (pq + pk) * (slice + 1) / a.slices;
    for (int pass = first; pass < last; ++pass) {
      const bool key = pass >= pq;
      const RopeTensor& t = a.t[key];
      const int head = (key ? pass - pq : pass) * per_pass + l.group;
      const bool in = head < t.heads;
      const int64_t at = (int64_t)head * a.dim;
      const int n0 = in ? l.n[0] : 0, n1 = in ? l.n[1] : 0;
      float x[2][8], w[2][8];
      if (!BWD || a.norm) {
        load_chunk((const T*)t.x + row * t.ldx + at + l.col[0], n0).get(x[0]);
        load_chunk((const T*)t.x + row * t.ldx + at + l.col[1], n1).get(x[1]);
      }
      if (a.norm && t.w) {
        load_chunk(t.w + l.col[0], n0).get(w[0]);
        load_chunk(t.w + l.col[1], n1).get(w[1]);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[0][j] = w[1][j] = 1.0f;
      }
      float r = 1.0f;
      if (a.norm) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) sq = fmaf(x[i][j], x[i][j], sq);
        sq = head_sum(sq, lanes);
        r = 1.0f / sqrtf(sq / (float)a.dim + a.eps);
      }
      T* out = (T*)t.out + row * t.ldo + at;
      if constexpr (!BWD) {
        if (a.norm) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = x[i][j] * r * w[i][j];
        }
        if (a.freqs > 0) rope_turn<NEXT>(l, a.freqs, x, cs, sn, 1.0f);
        store_chunk(out + l.col[0], n0, x[0]);
        store_chunk(out + l.col[1], n1, x[1]);
      } else {
        float d[2][8];
        load_chunk((const T*)t.dy + row * t.lddy + at + l.col[0], n0).get(d[0]);
        load_chunk((const T*)t.dy + row * t.lddy + at + l.col[1], n1).get(d[1]);
        if (a.freqs > 0) rope_turn<NEXT>(l, a.freqs, d, cs, sn, -1.0f);
        if (a.norm) {
          float dot = 0.0f;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              x[i][j] *= r;
              if (in) sum[key][i][j] = fmaf(d[i][j], x[i][j], sum[key][i][j]);
              d[i][j] *= w[i][j];
              dot = fmaf(d[i][j], x[i][j], dot);
            }
          dot = head_sum(dot, lanes) / (float)a.dim;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) d[i][j] = r * (d[i][j] - x[i][j] * dot);
        }
        store_chunk(out + l.col[0], n0, d[0]);
        store_chunk(out + l.col[1], n1, d[1]);
      }
    }
  }
  if constexpr (BWD) {
    if (!a.part) return;
#pragma unroll
    for (int key = 0; key < 2; ++key)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float v = sum[key][i][j];
          for (int o = lanes; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
          if (l.group == 0 && j < l.n[i]) s_sum[wave][key][l.col[i] + j] = v;
        }
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * a.dim; e += 256) {
      const int key = e / a.dim, d = e - key * a.dim;
      a.part[(int64_t)blockIdx.x * 2 * a.dim + e] = (s_sum[0][key][d] + s_sum[1][key][d]) + (s_sum[2][key][d] + s_sum[3][key][d]);
    }
  }
}

// Any head width up to 256 and any number of pairs: a wavefront takes a head of a token, a lane every 64th feature and reads its
// partner's beside it.
template <typename T, bool NEXT, bool BWD>
__global__ __launch_bounds__(256) void k_rope_any(RopeArgs a) {
  __shared__ float s_sum[BWD ? 4 : 1][2][BWD ? kRopeMostDim : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int heads = a.t[0].heads + a.t[1].heads;
  const int64_t items = a.rows * heads;
  float sum[2][4] = {};
  for (int64_t item = (int64_t)blockIdx.x * 4 + wave; item < items; item += (int64_t)gridDim.x * 4) {
    const int64_t row = item / heads;
    int head = (int)(item - row * heads);
    const bool key = head >= a.t[0].heads;
    if (key) head -= a.t[0].heads;
    const RopeTensor& t = a.t[key];
    const T* x = (const T*)t.x + row * t.ldx + (int64_t)head * a.dim;
    const T* dy = (const T*)t.dy + row * t.lddy + (int64_t)head * a.dim;
    T* out = (T*)t.out + row * t.ldo + (int64_t)head * a.dim;
    float v[4], u[4], cs[4], sn[4];                  // elements, partners, rotation (its sign in the sine)
    float xv[4], sq = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      v[i] = u[i] = xv[i] = sn[i] = 0.0f;
      cs[i] = 1.0f;
      if (e >= a.dim) continue;
      const int f = a.freqs, mate = e >= 2 * f ? e : NEXT ? e ^ 1 : e < f ? e + f : e - f;
      const T* from = BWD ? dy : x;
      v[i] = load_as_f32<T>(from, e);
      u[i] = load_as_f32<T>(from, mate);
      xv[i] = BWD ? (a.norm ? load_as_f32<T>(x, e) : 0.0f) : v[i];
      if (e < 2 * f) {
        const float2 c = turn_of(a, row, NEXT ? e >> 1 : e < f ? e : e - f);
        const bool lower = NEXT ? !(e & 1) : e < f;
        cs[i] = c.x;
        sn[i] = lower != BWD ? -c.y : c.y;
      }
      if (!BWD && a.norm && t.w) {
        v[i] *= t.w[e];
        u[i] *= t.w[mate];
      }
      sq = fmaf(xv[i], xv[i], sq);
    }
    const float r = a.norm ? 1.0f / sqrtf(wave_sum(sq) / (float)a.dim + a.eps) : 1.0f;
    float dot = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = lane + 64 * i;
      if (!BWD) {
        v[i] = e < 2 * a.freqs ? (v[i] * r) * cs[i] + (u[i] * r) * sn[i] : v[i] * r;
      } else {
        if (e < 2 * a.freqs) v[i] = v[i] * cs[i] + u[i] * sn[i];
        if (a.norm && e < a.dim) {
          xv[i] *= r;
          sum[key][i] = fmaf(v[i], xv[i], sum[key][i]);
          if (t.w) v[i] *= t.w[e];
          dot = fmaf(v[i], xv[i], dot);
        }
      }
    }
    if (BWD && a.norm) {
      dot = wave_sum(dot) / (float)a.dim;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = r * (v[i] - xv[i] * dot);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.dim) out[lane + 64 * i] = from_f32<T>(v[i]);
  }
  if constexpr (BWD) {
    if (!a.part) return;
#pragma unroll
    for (int key = 0; key < 2; ++key)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < a.dim) s_sum[wave][key][lane + 64 * i] = sum[key][i];
    __syncthreads();
    for (int e = threadIdx.x; e < 2 * a.dim; e += 256) {
      const int key = e / a.dim, d = e - key * a.dim;
      a.part[(int64_t)blockIdx.x * 2 * a.dim + e] = (s_sum[0][key][d] + s_sum[1][key][d]) + (s_sum[2][key][d] + s_sum[3][key][d]);
    }
  }
}

// the blocks' sums put together, in fixed order and fp64: 16 columns a block, 16 lanes each
__global__ __launch_bounds__(256) void k_rope_finish(const float* __restrict__ part, int blocks, int dim, float* __restrict__ dwq,
                                                     float* __restrict__ dwk) {
  __shared__ double red[16][17];
  const int c = threadIdx.x & 15, s = threadIdx.x >> 4, e = blockIdx.x * 16 + c;
  double v = 0.0;
  if (e < 2 * dim)
    for (int b = s; b < blocks; b += 16) v += part[(int64_t)b * 2 * dim + e];
  red[s][c] = v;
  __syncthreads();
  if (s == 0 && e < 2 * dim) {
    for (int i = 1; i < 16; ++i) v += red[i][c];
    float* to = e < dim ? dwq : dwk;
    if (to) to[e < dim ? e : e - dim] = (float)v;
  }
}

// lanes of a head in k_rope; 0: k_rope_any
static int rope_lanes(int64_t dim, int64_t freqs, int neighbours) {
  if (dim % 8 || (!neighbours && freqs % 8)) return 0;
  int lanes = 1;
  while (lanes * 16 < dim) lanes *= 2;
  return lanes;
}
constexpr int64_t kRopeBlocks = 1024;                // of a backward pass at most: four a CU
static int64_t rope_bwd_blocks(int64_t rows, int64_t heads) {
  const int64_t b = ceil_div(rows * heads, 4);
  return b < kRopeBlocks ? b : kRopeBlocks;
}
// slices of a token's heads: enough wavefronts for the chip where there are few tokens
static int rope_slices(int64_t rows, int passes) {
  const int64_t want = ceil_div(4096, rows);
  return (int)(want < passes ? want : passes);
}

static int rope_args(RopeArgs* a, int dtype, int64_t T, int64_t heads, int64_t kv_heads, int64_t dim, int norm, float eps, const int32_t* pos,
                     int64_t axes, const int32_t* axis, const float* inv_freq, int64_t freqs, int neighbours) {
  if (T <= 0 || T > (INT64_C(1) << 28) || heads <= 0 || kv_heads < 0 || heads + kv_heads > 65535 || dim <= 0 || dim > kRopeMostDim || freqs < 0 ||
      2 * freqs > dim || axes < 0 || axes > 16 || !(eps >= 0.0f) || !(eps < INFINITY))
    return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if ((norm != 0 && norm != 1) || (neighbours != 0 && neighbours != 1)) return EFQAT_ERR_BAD_LAYOUT;
  if (freqs > 0 && axes < 1) return EFQAT_ERR_BAD_SHAPE;
  if (freqs > 0 && (!pos || !inv_freq || (axes > 1 && !axis))) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(pos) || !aligned4(axis) || !aligned4(inv_freq)) return EFQAT_ERR_ALIGNMENT;
  a->rows = T;
  a->dim = (int)dim;
  a->freqs = (int)freqs;
  a->axes = (int)axes;
  a->norm = norm;
  a->pos = pos;
  a->axis = axes > 1 ? axis : nullptr;
  a->inv_freq = inv_freq;
  a->eps = eps;
  a->part = nullptr;
  a->slices = 1;
  return EFQAT_OK;
}
static int rope_rows(const void* p, int64_t ld, int64_t cols, int dtype) {
  if (ld < cols) return EFQAT_ERR_BAD_SHAPE;
  if (!p) return EFQAT_ERR_NULL_PTR;
  return aligned_for(p, dtype) ? EFQAT_OK : EFQAT_ERR_ALIGNMENT;
}
template <bool BWD>
static int rope_launch(RopeArgs& a, int dtype, int neighbours, unsigned* blocks, hipStream_t st) {
  const int lanes = rope_lanes(a.dim, a.freqs, neighbours), heads = a.t[0].heads + a.t[1].heads;
  if (lanes) {
    const int per_pass = 64 / lanes, passes = (int)(ceil_div(a.t[0].heads, per_pass) + ceil_div(a.t[1].heads, per_pass));
    a.slices = rope_slices(a.rows, passes);
  }
  const int64_t need = ceil_div(lanes ? a.rows * a.slices : a.rows * heads, 4);
  const int64_t most = BWD ? rope_bwd_blocks(a.rows, heads) : 1 << 23;          // a grid has fewer than 2^32 lanes
  const unsigned n = *blocks = (unsigned)(need < most ? need : most);
#define EFQAT_ROPE(E, NEXT)                                                                       \
  do {                                                                                            \
    if (lanes) return launch(k_rope<E, NEXT, BWD>, dim3(n), dim3(256), 0, st, a, lanes);          \
    return launch(k_rope_any<E, NEXT, BWD>, dim3(n), dim3(256), 0, st, a);                        \
  } while (0)
  if (dtype == EFQAT_F32) { if (neighbours) EFQAT_ROPE(float, true); EFQAT_ROPE(float, false); }
  if (neighbours) EFQAT_ROPE(bf16_t, true);
  EFQAT_ROPE(bf16_t, false);
#undef EFQAT_ROPE
}

}  // namespace efqat

using namespace efqat;

extern "C" int efqat_head_norm_rope_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, int dtype, int64_t T, int64_t heads,
                                        int64_t kv_heads, int64_t dim, int norm, const float* q_weight, const float* k_weight, float eps,
                                        const int32_t* positions, int64_t axes, const int32_t* axis, const float* inv_freq, int64_t freqs,
                                        int neighbours, void* yq, int64_t ldyq, void* yk, int64_t ldyk, void* stream) {
  RopeArgs a;
  EFQAT_TRY(rope_args(&a, dtype, T, heads, kv_heads, dim, norm, eps, positions, axes, axis, inv_freq, freqs, neighbours));
  EFQAT_TRY(rope_rows(q, ldq, heads * dim, dtype));
  EFQAT_TRY(rope_rows(yq, ldyq, heads * dim, dtype));
  if (kv_heads > 0) {
    EFQAT_TRY(rope_rows(k, ldk, kv_heads * dim, dtype));
    EFQAT_TRY(rope_rows(yk, ldyk, kv_heads * dim, dtype));
  }
  if (!aligned4(q_weight) || !aligned4(k_weight)) return EFQAT_ERR_ALIGNMENT;
  a.t[0] = {q, nullptr, yq, ldq, 0, ldyq, q_weight, (int)heads};
  a.t[1] = {k, nullptr, yk, ldk, 0, ldyk, k_weight, (int)kv_heads};
  unsigned blocks;
  return rope_launch<false>(a, dtype, neighbours, &blocks, (hipStream_t)stream);
}

extern "C" size_t efqat_head_norm_rope_bwd_workspace_bytes(int64_t T, int64_t heads, int64_t kv_heads, int64_t dim) {
  if (T <= 0 || T > (INT64_C(1) << 28) || heads <= 0 || kv_heads < 0 || heads + kv_heads > 65535 || dim <= 0 || dim > kRopeMostDim) return 256;
  return (size_t)round_up(rope_bwd_blocks(T, heads + kv_heads) * 2 * dim * 4, 256);
}

extern "C" int efqat_head_norm_rope_bwd(const void* dyq, int64_t lddyq, const void* dyk, int64_t lddyk, const void* q, int64_t ldq, const void* k,
                                        int64_t ldk, int dtype, int64_t T, int64_t heads, int64_t kv_heads, int64_t dim, int norm,
                                        const float* q_weight, const float* k_weight, float eps, const int32_t* positions, int64_t axes,
                                        const int32_t* axis, const float* inv_freq, int64_t freqs, int neighbours, void* dq, int64_t lddq,
                                        void* dk, int64_t lddk, float* dq_weight, float* dk_weight, void* ws, size_t ws_bytes, void* stream) {
  RopeArgs a;
  EFQAT_TRY(rope_args(&a, dtype, T, heads, kv_heads, dim, norm, eps, positions, axes, axis, inv_freq, freqs, neighbours));
  EFQAT_TRY(rope_rows(dyq, lddyq, heads * dim, dtype));
  EFQAT_TRY(rope_rows(dq, lddq, heads * dim, dtype));
  if (norm) EFQAT_TRY(rope_rows(q, ldq, heads * dim, dtype));
  if (kv_heads > 0) {
    EFQAT_TRY(rope_rows(dyk, lddyk, kv_heads * dim, dtype));
    EFQAT_TRY(rope_rows(dk, lddk, kv_heads * dim, dtype));
    if (norm) EFQAT_TRY(rope_rows(k, ldk, kv_heads * dim, dtype));
  }
  if (!norm && (dq_weight || dk_weight)) return EFQAT_ERR_BAD_LAYOUT;
  if (!aligned4(q_weight) || !aligned4(k_weight) || !aligned4(dq_weight) || !aligned4(dk_weight)) return EFQAT_ERR_ALIGNMENT;
  const bool sums = dq_weight || dk_weight;
  if (sums) {
    if (!ws) return EFQAT_ERR_NULL_PTR;
    if ((uintptr_t)ws % 256) return EFQAT_ERR_ALIGNMENT;
    if (ws_bytes < efqat_head_norm_rope_bwd_workspace_bytes(T, heads, kv_heads, dim)) return EFQAT_ERR_WORKSPACE;
    a.part = (float*)ws;
  }
  a.t[0] = {q, dyq, dq, ldq, lddyq, lddq, q_weight, (int)heads};
  a.t[1] = {k, dyk, dk, ldk, lddyk, lddk, k_weight, (int)kv_heads};
  unsigned blocks;
  hipStream_t st = (hipStream_t)stream;
  EFQAT_TRY(rope_launch<true>(a, dtype, neighbours, &blocks, st));
  if (!sums) return EFQAT_OK;
  return launch(k_rope_finish, dim3((unsigned)ceil_div(2 * dim, 16)), dim3(256), 0, st, (const float*)a.part, (int)blocks, (int)dim, dq_weight,
                kv_heads > 0 ? dk_weight : nullptr);
}
