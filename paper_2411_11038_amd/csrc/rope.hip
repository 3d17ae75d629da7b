// Norms of queries and keys for each head with the position rotation in the same pass, forward and backward.
//
//   r = 1 / sqrt(mean_d x_d^2 + eps),  xhat = x r,  n = xhat w
//   y_a = n_a cos t - n_b sin t,  y_b = n_b cos t + n_a sin t  for the F pairs (a, b) of a head,  t = pos[axis(j)] f_j;  y = n behind them
//   dn = the rotation back of dy,  g = dn w,  dx = r (g - xhat mean_d (g xhat)),  dw_d = sum over tokens and heads of dn_d xhat_d
//
// Bound by HBM: what is read is written once.  A lane owns two chunks of 8 features that hold both members of their pairs, so that the
// rotation stays in the lane and the norm is a sum over the D / 16 lanes of a head.  A wavefront takes a token: it makes the F angles
// once (the product in 64 bits, its whole turns taken off, so that far positions keep their place in the circle) and walks the heads, the next
// ones on their way.  bf16, 8192 tokens, 32 + 8 heads of 128, backward: 50 us (252 MB, 5.0 TB/s) and 6 us for the sums of the weights' gradients, fp32
// 140 us in all (503 MB); fp32, 4099
// tokens, 24 heads of 80, three axes, forward: 19 us (63 MB), where three lanes of eight have no features; 16 tokens: 4 us of kernel in a call of 6.2.
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
  int dim, freqs, axes, norm;
  const int32_t* pos;                                // [axes][rows]
  const int32_t* axis;
  const float* inv_freq;
  float eps;
  float* part;                                       // backward: [blocks][dim] sums of dn xhat
};

// a pair's position and frequency
struct Angle {
  int pos;
  float f;
  __device__ __forceinline__ Angle() {}
  __device__ __forceinline__ Angle(const RopeArgs& a, int64_t row, int j) {
    int ax = a.axis ? a.axis[j] : 0;
    ax = ax < 0 ? 0 : ax >= a.axes ? a.axes - 1 : ax;
    pos = a.pos[ax * a.rows + row];
    f = a.inv_freq[j];
  }
  // cosine and sine: the turns are formed in 64 bits, their fraction is exact to 2^-25
  __device__ __forceinline__ float2 turn() const {
    const double turns = (double)pos * (double)f * 0.15915494309189533577;
    float2 cs;
    sincospif((float)(2.0 * (turns - rint(turns))), &cs.y, &cs.x);
    return cs;
  }
};

constexpr int kRopeMostDim = 256;
constexpr int kRopeBlocks = 1024;                    // of a backward pass at most: four a CU

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
// Rotation (sign 1) or rotation back (-1) of a lane's 16 elements; what has no pair stays as it is, whatever lies beside it.  The turns of a
// token's pairs are read from LDS each time: lanes have more heads' registers to fill.
template <bool NEXT>
__device__ __forceinline__ void rope_turn(const RopeLane& l, int freqs, float (&v)[2][8], const float2* turns, float sign) {
  if constexpr (NEXT) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = l.pair + 4 * i + j < freqs;
        const float2 cs = turns[l.pair + 4 * i + j];
        const float x = v[i][2 * j], y = v[i][2 * j + 1], s = sign * cs.y;
        v[i][2 * j] = in ? x * cs.x - y * s : x;
        v[i][2 * j + 1] = in ? y * cs.x + x * s : y;
      }
  } else if (l.turned) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float2 cs = turns[l.pair + j];
      const float x = v[0][j], y = v[1][j], s = sign * cs.y;
      v[0][j] = x * cs.x - y * s;
      v[1][j] = y * cs.x + x * s;
    }
  }
}
// sum over the lanes of a head
__device__ __forceinline__ float head_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// How the work is laid out: a wavefront takes a token's queries or its keys, `per` passes of them at most (a pass: 64 / lanes heads).  The first
// blocks have the queries' units, the others the keys'; backward blocks walk theirs and keep the weights' sums.
struct RopeUnits {
  int lanes, per, passes[2], units[2];               // passes of a token, units they are cut into
  int blocks[2];
};

template <typename T, bool NEXT, bool BWD>
__global__ __launch_bounds__(256, BWD ? 4 : 5) void k_rope(RopeArgs a, RopeUnits u) {
  __shared__ float2 s_turn[4][kRopeMostDim / 2];
  __shared__ float s_sum[BWD ? 4 : 1][BWD ? kRopeMostDim : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const RopeLane l = rope_lane<NEXT>(a, u.lanes);
  const int key = (int)blockIdx.x >= u.blocks[0], per_pass = 64 / u.lanes, units = u.units[key];
  const RopeTensor& t = a.t[key];
  const int64_t items = a.rows * units;
  float w[2][8], sum[2][8] = {};
  if (a.norm && t.w) {
    load_chunk(t.w + l.col[0], l.n[0]).get(w[0]);
    load_chunk(t.w + l.col[1], l.n[1]).get(w[1]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[0][j] = w[1][j] = 1.0f;
  }
  const float inv_dim = 1.0f / (float)a.dim;
  for (int64_t item = (int64_t)(blockIdx.x - (key ? u.blocks[0] : 0)) * 4 + wave; item < items; item += (int64_t)u.blocks[key] * 4) {
    const int64_t row = item / units;
    const int unit = (int)(item - row * units), first = unit * u.per, last = min(first + u.per, u.passes[key]);
    const T* const x_row = (const T*)t.x + row * t.ldx;
    const T* const dy_row = (const T*)t.dy + row * t.lddy;
    T* const out_row = (T*)t.out + row * t.ldo;
    Raw8<T> rx[2], rd[2];
    auto load = [&](int pass) {
      const int head = pass * per_pass + l.group;
      const int64_t at = (int64_t)head * a.dim;
      const bool in = head < t.heads;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int n = in ? l.n[i] : 0;
        if (!BWD || a.norm) rx[i] = load_chunk(x_row + at + l.col[i], n);
        if constexpr (BWD) rd[i] = load_chunk(dy_row + at + l.col[i], n);
      }
    };
    // what the angles are made of is asked for first, the first heads are on their way while they are made
    Angle angle[2];
    if (lane < a.freqs) angle[0] = Angle(a, row, lane);
    if (lane + 64 < a.freqs) angle[1] = Angle(a, row, lane + 64);
    load(first);
    if (a.freqs > 0) {
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // the item before has read its turns
      __builtin_amdgcn_wave_barrier();
      if (lane < a.freqs) s_turn[wave][lane] = angle[0].turn();
      if (lane + 64 < a.freqs) s_turn[wave][lane + 64] = angle[1].turn();
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
    for (int pass = first; pass < last; ++pass) {
      const int head = pass * per_pass + l.group;
      const bool in = head < t.heads;
      float x[2][8], d[2][8], r = 1.0f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (!BWD || a.norm) rx[i].get(x[i]);
        if constexpr (BWD) rd[i].get(d[i]);
      }
      if (pass + 1 < last) load(pass + 1);
      if (a.norm) {
        float sq = 0.0f;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int j = 0; j < 8; ++j) sq = fmaf(x[i][j], x[i][j], sq);
        r = 1.0f / sqrtf(fmaf(head_sum(sq, u.lanes), inv_dim, a.eps));
        if (BWD && !in) r = 0.0f;                    // no head: without eps 1 / 0, and its zeros would be NaN in the weights' sums
      }
      if constexpr (!BWD) {
        if (a.norm) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] = x[i][j] * r * w[i][j];
        }
        if (a.freqs > 0) rope_turn<NEXT>(l, a.freqs, x, s_turn[wave], 1.0f);
      } else {
        if (a.freqs > 0) rope_turn<NEXT>(l, a.freqs, d, s_turn[wave], -1.0f);
        if (a.norm) {
          float dot = 0.0f;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              x[i][j] *= r;                          // of a head that does not exist: zeros
              sum[i][j] = fmaf(d[i][j], x[i][j], sum[i][j]);
              d[i][j] *= w[i][j];
              dot = fmaf(d[i][j], x[i][j], dot);
            }
          dot = head_sum(dot, u.lanes) * inv_dim;
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) d[i][j] = r * (d[i][j] - x[i][j] * dot);
        }
      }
      const int64_t at = (int64_t)head * a.dim;
#pragma unroll
      for (int i = 0; i < 2; ++i) store_chunk(out_row + at + l.col[i], in ? l.n[i] : 0, BWD ? d[i] : x[i]);
    }
  }
  if constexpr (BWD) {
    if (!a.part) return;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float v = sum[i][j];
        for (int o = u.lanes; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
        if (l.group == 0 && j < l.n[i]) s_sum[wave][l.col[i] + j] = v;
      }
    __syncthreads();
    for (int d = threadIdx.x; d < a.dim; d += 256)
      a.part[(int64_t)blockIdx.x * a.dim + d] = (s_sum[0][d] + s_sum[1][d]) + (s_sum[2][d] + s_sum[3][d]);
  }
}

// Any head width up to 256 and any number of pairs: a wavefront takes a head of a token, a lane every 64th feature and reads its
// partner's beside it.  Turns are made anew for every head and both members of a pair, and loads are one element a lane: 8192 tokens, 12 + 12 heads of 80
// with 20 pairs, bf16 81 us forward and 129 backward where k_rope (neighbours paired) takes 19.5 and 34; fp32 88 and 151.
template <typename T, bool NEXT, bool BWD>
__global__ __launch_bounds__(256) void k_rope_any(RopeArgs a, RopeUnits u) {
  __shared__ float s_sum[BWD ? 4 : 1][BWD ? kRopeMostDim : 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int key = (int)blockIdx.x >= u.blocks[0];
  const RopeTensor& t = a.t[key];
  const int heads = t.heads;
  const int64_t items = a.rows * heads;
  float sum[4] = {};
  for (int64_t item = (int64_t)(blockIdx.x - (key ? u.blocks[0] : 0)) * 4 + wave; item < items; item += (int64_t)u.blocks[key] * 4) {
    const int64_t row = item / heads;
    const int head = (int)(item - row * heads);
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
        const float2 c = Angle(a, row, NEXT ? e >> 1 : e < f ? e : e - f).turn();
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
          sum[i] = fmaf(v[i], xv[i], sum[i]);
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
    for (int i = 0; i < 4; ++i)
      if (lane + 64 * i < a.dim) s_sum[wave][lane + 64 * i] = sum[i];
    __syncthreads();
    for (int d = threadIdx.x; d < a.dim; d += 256)
      a.part[(int64_t)blockIdx.x * a.dim + d] = (s_sum[0][d] + s_sum[1][d]) + (s_sum[2][d] + s_sum[3][d]);
  }
}

// The blocks' sums put together, in fixed order and fp64: four columns a block, 64 lanes each; the queries' first, then the keys'.
__global__ __launch_bounds__(256) void k_rope_finish(const float* __restrict__ part, RopeUnits u, int dim, float* __restrict__ dwq,
                                                     float* __restrict__ dwk) {
  __shared__ double red[4][4];
  const int key = blockIdx.y, c = threadIdx.x & 3, s = threadIdx.x >> 2, e = blockIdx.x * 4 + c, blocks = u.blocks[key];
  const float* from = part + (key ? (int64_t)u.blocks[0] * dim : 0);
  float* to = key ? dwk : dwq;
  if (!to) return;
  double v = 0.0;
  if (e < dim) {
    float x[kRopeBlocks / 64];
#pragma unroll
    for (int b = 0; b < kRopeBlocks / 64; ++b) x[b] = s + 64 * b < blocks ? from[(int64_t)(s + 64 * b) * dim + e] : 0.0f;
#pragma unroll
    for (int b = 0; b < kRopeBlocks / 64; ++b) v += x[b];
  }
#pragma unroll
  for (int o = 4; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
  if ((threadIdx.x & 63) < 4) red[threadIdx.x >> 6][c] = v;
  __syncthreads();
  if (threadIdx.x < 4 && e < dim) to[e] = (float)((red[0][c] + red[1][c]) + (red[2][c] + red[3][c]));
}

// lanes of a head in k_rope; 0: k_rope_any
static int rope_lanes(int64_t dim, int64_t freqs, int neighbours) {
  if (dim % 8 || (!neighbours && freqs % 8)) return 0;
  int lanes = 1;
  while (lanes * 16 < dim) lanes *= 2;
  return lanes;
}
// Units and blocks of a call.  Few tokens: a pass a wavefront; else four, whose loads follow each other.  One pass and four, 32 + 8 heads of 128 (five
// passes a token), us: forward bf16 1024 tokens 7.5 and 8.3, 2048 10.9 and 9.5, 4096 16.9 and 14.8, 8192 35.1 and 30.8, fp32 4096 30.0 and 30.4; backward
// bf16 2048 24.5 and 21.5, 4096 34.0 and 36.1, 8192 53.5 and 60.0 (four loses there, whose blocks walk the tokens anyway), fp32 2048 49.0 and 42.5,
// 8192 140.9 and 139.7.
static RopeUnits rope_units(int64_t rows, int64_t heads, int64_t kv_heads, int lanes, bool bwd) {
  RopeUnits u = {};
  u.lanes = lanes;
  const int64_t n[2] = {heads, kv_heads};
  int64_t need[2], all = 0;
  for (int i = 0; i < 2; ++i) {
    u.passes[i] = (int)(lanes ? ceil_div(n[i], 64 / lanes) : n[i]);
    all += u.passes[i];
  }
  u.per = lanes && rows * all > 16384 ? 4 : 1;
  all = 0;
  for (int i = 0; i < 2; ++i) {
    u.units[i] = (int)ceil_div(u.passes[i], u.per);
    need[i] = ceil_div(rows * u.units[i], 4);
    all += need[i];
  }
  const int64_t most = bwd ? kRopeBlocks : 1 << 23;                  // a grid has fewer than 2^32 lanes
  for (int i = 0; i < 2; ++i) {
    // shared out by the passes that there are, at least one each
    const int64_t part = all <= most ? need[i] : need[i] == 0 ? 0 : (most - 1) * u.passes[i] / (u.passes[0] + u.passes[1]) + (i == 1);
    u.blocks[i] = (int)(part < 1 && need[i] > 0 ? 1 : part < need[i] ? part : need[i]);
  }
  return u;
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
  return EFQAT_OK;
}
static int rope_rows(const void* p, int64_t ld, int64_t cols, int dtype) {
  if (ld < cols) return EFQAT_ERR_BAD_SHAPE;
  if (!p) return EFQAT_ERR_NULL_PTR;
  return aligned_for(p, dtype) ? EFQAT_OK : EFQAT_ERR_ALIGNMENT;
}
template <bool BWD>
static int rope_launch(const RopeArgs& a, const RopeUnits& u, int dtype, int neighbours, hipStream_t st) {
  const dim3 grid((unsigned)(u.blocks[0] + u.blocks[1]));
#define EFQAT_ROPE(E, NEXT)                                                            \
  do {                                                                                 \
    if (u.lanes) return launch(k_rope<E, NEXT, BWD>, grid, dim3(256), 0, st, a, u);    \
    return launch(k_rope_any<E, NEXT, BWD>, grid, dim3(256), 0, st, a, u);             \
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
  const RopeUnits u = rope_units(T, heads, kv_heads, rope_lanes(dim, freqs, neighbours), false);
  return rope_launch<false>(a, u, dtype, neighbours, (hipStream_t)stream);
}

extern "C" size_t efqat_head_norm_rope_bwd_workspace_bytes(int64_t T, int64_t heads, int64_t kv_heads, int64_t dim) {
  if (T <= 0 || T > (INT64_C(1) << 28) || heads <= 0 || kv_heads < 0 || heads + kv_heads > 65535 || dim <= 0 || dim > kRopeMostDim) return 256;
  return (size_t)round_up(kRopeBlocks * dim * 4, 256);
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
  const RopeUnits u = rope_units(T, heads, kv_heads, rope_lanes(dim, freqs, neighbours), true);
  hipStream_t st = (hipStream_t)stream;
  EFQAT_TRY(rope_launch<true>(a, u, dtype, neighbours, st));
  if (!sums) return EFQAT_OK;
  return launch(k_rope_finish, dim3((unsigned)ceil_div(dim, 4), kv_heads > 0 ? 2 : 1), dim3(256), 0, st, (const float*)a.part, u, (int)dim, dq_weight,
                dk_weight);
}
