// The activation of a feed-forward block, y = f(x) or y = f(x) u, and the 8-bit checkpoint that keeps its inputs for the
// backward pass.  f is x Phi(x) (GELU) or x / (1 + exp(-x)) (SiLU).
//
// One pass over the data each way, bound by HBM: a lane owns 8 neighbouring columns, 16 lanes the 128 columns that share a
// scale, so that a group's largest magnitude is four DPP steps away and neither LDS nor a second read is needed.  What is read
// is written once: y and the codes leave in the pass that reads x and u.
//
// bf16, 8192 x 11008, gated: forward with both inputs kept 135 us (726 MB, 5.4 TB/s; a copy of 1 GiB reaches 5.0, of 256 MiB 5.4),
// backward 124 us (726 MB, 5.8 TB/s), a checkpoint read back 53 us (273 MB, 5.2 TB/s).  Small calls are a launch: 16 x 11008 forward
// 2.6 us of kernel in 4.8 us a call.  fp32 2049 x 1001, rows of any alignment, backward 5.9 us (18 MB).  GELU of one input in bf16 is bound by
// its operations beside the bytes: 8192 x 11008 forward 84 us (361 MB, 4.3 TB/s).
#include "rows.hpp"

namespace efqat {

// exp(-x^2 / 2) and the tail Phi(-|x|) from it: Phi(-a) exp(a^2 / 2) = t Q(t), t = 1 / (1 + 0.43 a / sqrt(2)).  Q, of degree 7, is fitted to
// the smallest largest relative error over 0 <= a <= 13.7 (8.9e-8), behind which the exponential leaves fp32: the tail of a negative x
// keeps its digits, however far out, and is not the difference of two numbers near 1.  One exponential serves the value and the slope.
// What is lost in its argument, up to 2^-24 of 92, is put back where the results are fp32.
template <bool FINE>
__device__ __forceinline__ float gelu_tail(float x, float* gauss) {
  const float a = FINE ? fminf(fabsf(x), 32.0f) : fabsf(x);     // the same exponential, 0, from there on: what is put back stays finite
  const float b = -0.5f * a, h = a * b, s = h * 1.4426950408889634f;
  float e = __builtin_amdgcn_exp2f(s);
  if constexpr (FINE) e = fmaf(e, fmaf(-s, 0.69314718055994531f, h) + fmaf(a, b, -h), e);
  *gauss = e;
  const float t = __builtin_amdgcn_rcpf(fmaf(0.30405591591021547f, a, 1.0f));
  float q = fmaf(3.676769939e-02f, t, -1.548372005e-01f);
  q = fmaf(q, t, 1.912668004e-01f);
  q = fmaf(q, t, -4.233731386e-02f);
  q = fmaf(q, t, 1.231508887e-01f);
  q = fmaf(q, t, 1.025559401e-01f);
  q = fmaf(q, t, 1.221750987e-01f);
  q = fmaf(q, t, 1.212581128e-01f);
  return q * t * e;
}
template <int KIND, bool FINE>
__device__ __forceinline__ float act_value(float x) {
  if constexpr (KIND == EFQAT_ACT_GELU) {
    float e;
    const float q = gelu_tail<FINE>(x, &e);
    return x * (x >= 0.0f ? 1.0f - q : q);
  } else {
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
  }
}
// f(x) and f'(x)
template <int KIND, bool FINE>
__device__ __forceinline__ float act_slope(float x, float* value) {
  if constexpr (KIND == EFQAT_ACT_GELU) {
    float e;
    const float q = gelu_tail<FINE>(x, &e);
    const float phi = x >= 0.0f ? 1.0f - q : q;
    *value = x * phi;
    return fmaf(x * 0.39894228040143268f, e, phi);
  } else {
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.4426950408889634f));
    *value = x * s;
    return fmaf(*value, 1.0f - s, s);
  }
}

// Group of 128 columns that 16 lanes take: 16 groups a block, numbered along the rows.  n: columns of the lane's chunk (<= 0:
// none), pad: the chunk lies inside the pitch of the codes.
struct GroupPlace {
  int64_t row, group, col;
  int n;
  bool in, pad;
};
__device__ __forceinline__ GroupPlace group_place(int64_t rows, int64_t cols, uint32_t gpr) {
  const uint64_t first = (uint64_t)blockIdx.x * 16;
  const uint64_t row0 = first / gpr;
  const uint32_t at = (uint32_t)(first - row0 * gpr) + (threadIdx.x >> 4);      // gpr < 2^31: see check_rows
  GroupPlace g;
  const uint32_t more = at / gpr;
  g.row = (int64_t)row0 + more;
  g.in = g.row < rows;
  g.group = at - more * gpr;
  g.col = g.group * kCkptGroup + (threadIdx.x & 15) * 8;
  const int64_t left = g.in ? cols - g.col : 0;
  g.n = left > 8 ? 8 : (int)(left < 0 ? 0 : left);
  g.pad = g.in && g.col < ckpt_pitch(cols);
  return g;
}

struct Ckpt {
  int8_t* codes;
  float* scales;
};
__device__ __forceinline__ void ckpt_write(const Ckpt& k, const GroupPlace& g, int64_t cols, uint32_t gpr, const float (&v)[8]) {
  float scale;
  const uint2 q = ckpt_encode(v, &scale);
  if (g.pad) *reinterpret_cast<uint2*>(k.codes + g.row * ckpt_pitch(cols) + g.col) = q;
  if (g.in && (threadIdx.x & 15) == 0) k.scales[g.row * gpr + g.group] = scale;
}
__device__ __forceinline__ void ckpt_read(const Ckpt& k, const GroupPlace& g, int64_t cols, uint32_t gpr, float (&v)[8]) {
  const uint2 q = *reinterpret_cast<const uint2*>(k.codes + g.row * ckpt_pitch(cols) + g.col);
  ckpt_decode(q, k.scales[g.row * gpr + g.group], v);
}

template <typename T>
__global__ __launch_bounds__(256) void k_ckpt_save(const T* __restrict__ x, int64_t ldx, int64_t rows, int64_t cols, uint32_t gpr, Ckpt k) {
  const GroupPlace g = group_place(rows, cols, gpr);
  float v[8];
  load_chunk(x + g.row * ldx + g.col, g.n).get(v);
  ckpt_write(k, g, cols, gpr, v);
}

template <typename T>
__global__ __launch_bounds__(256) void k_ckpt_load(Ckpt k, int64_t rows, int64_t cols, uint32_t gpr, T* __restrict__ x, int64_t ldx) {
  const GroupPlace g = group_place(rows, cols, gpr);
  if (g.n <= 0) return;
  float v[8];
  ckpt_read(k, g, cols, gpr, v);
  store_chunk(x + g.row * ldx + g.col, g.n, v);
}

template <typename T, int KIND, bool GATED, bool KEEP>
__global__ __launch_bounds__(256) void k_act_fwd(const T* __restrict__ x, int64_t ldx, const T* __restrict__ u, int64_t ldu, int64_t rows,
                                                 int64_t cols, uint32_t gpr, T* __restrict__ y, int64_t ldy, Ckpt kx, Ckpt ku) {
  const GroupPlace g = group_place(rows, cols, gpr);
  Raw8<T> rx = load_chunk(x + g.row * ldx + g.col, g.n), ru;
  if constexpr (GATED) ru = load_chunk(u + g.row * ldu + g.col, g.n);
  float v[8], w[8], o[8];
  rx.get(v);
#pragma unroll
  for (int j = 0; j < 8; ++j) o[j] = act_value<KIND, sizeof(T) == 4>(v[j]);
  if constexpr (GATED) {
    ru.get(w);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] *= w[j];
  }
  store_chunk(y + g.row * ldy + g.col, g.n, o);
  if constexpr (KEEP) {
    ckpt_write(kx, g, cols, gpr, v);
    if constexpr (GATED) ckpt_write(ku, g, cols, gpr, w);
  }
}

template <typename T, int KIND, bool GATED>
__global__ __launch_bounds__(256) void k_act_bwd(const T* __restrict__ dy, int64_t lddy, int64_t rows, int64_t cols, uint32_t gpr, Ckpt kx,
                                                 Ckpt ku, T* __restrict__ dx, int64_t lddx, T* __restrict__ du, int64_t lddu) {
  const GroupPlace g = group_place(rows, cols, gpr);
  if (g.n <= 0) return;
  const Raw8<T> rd = load_chunk(dy + g.row * lddy + g.col, g.n);
  float v[8], w[8], d[8];
  ckpt_read(kx, g, cols, gpr, v);
  if constexpr (GATED) ckpt_read(ku, g, cols, gpr, w);
  rd.get(d);
  float a[8], b[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    float f;
    const float s = act_slope<KIND, sizeof(T) == 4>(v[j], &f);
    a[j] = d[j] * s;
    if constexpr (GATED) {
      a[j] *= w[j];
      b[j] = d[j] * f;
    }
  }
  store_chunk(dx + g.row * lddx + g.col, g.n, a);
  if constexpr (GATED) store_chunk(du + g.row * lddu + g.col, g.n, b);
}

// rows of an elementwise call and its grid of 16 groups a block
static int check_rows(int64_t rows, int64_t cols, unsigned* blocks) {
  if (rows <= 0 || cols <= 0 || rows > INT64_C(1) << 40 || cols > INT32_MAX) return EFQAT_ERR_BAD_SHAPE;
  const int64_t groups = ckpt_groups(cols);
  if (rows > (INT64_C(16) * INT32_MAX) / groups) return EFQAT_ERR_BAD_SHAPE;
  *blocks = (unsigned)ceil_div(rows * groups, 16);
  return EFQAT_OK;
}

}  // namespace efqat

using namespace efqat;

extern "C" int64_t efqat_ckpt8_pitch(int64_t cols) { return cols <= 0 ? 0 : ckpt_pitch(cols); }

extern "C" int efqat_ckpt8_save(const void* x, int64_t ldx, int dtype, int64_t rows, int64_t cols, int8_t* codes, float* scales,
                                void* stream) {
  unsigned blocks;
  if (const int rc = check_rows(rows, cols, &blocks)) return rc;
  if (ldx < cols) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (!x || !codes || !scales) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(x, dtype) || !aligned16(codes) || !aligned4(scales)) return EFQAT_ERR_ALIGNMENT;
  const uint32_t gpr = (uint32_t)ckpt_groups(cols);
  const Ckpt k = {codes, scales};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EFQAT_F32) EFQAT_TRY(launch(k_ckpt_save<float>, dim3(blocks), dim3(256), 0, st, (const float*)x, ldx, rows, cols, gpr, k));
  else EFQAT_TRY(launch(k_ckpt_save<bf16_t>, dim3(blocks), dim3(256), 0, st, (const bf16_t*)x, ldx, rows, cols, gpr, k));
  return EFQAT_OK;
}

extern "C" int efqat_ckpt8_load(const int8_t* codes, const float* scales, int64_t rows, int64_t cols, void* x, int64_t ldx, int dtype,
                                void* stream) {
  unsigned blocks;
  if (const int rc = check_rows(rows, cols, &blocks)) return rc;
  if (ldx < cols) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (!x || !codes || !scales) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(x, dtype) || !aligned16(codes) || !aligned4(scales)) return EFQAT_ERR_ALIGNMENT;
  const uint32_t gpr = (uint32_t)ckpt_groups(cols);
  const Ckpt k = {const_cast<int8_t*>(codes), const_cast<float*>(scales)};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EFQAT_F32) EFQAT_TRY(launch(k_ckpt_load<float>, dim3(blocks), dim3(256), 0, st, k, rows, cols, gpr, (float*)x, ldx));
  else EFQAT_TRY(launch(k_ckpt_load<bf16_t>, dim3(blocks), dim3(256), 0, st, k, rows, cols, gpr, (bf16_t*)x, ldx));
  return EFQAT_OK;
}

extern "C" int efqat_act_fwd(const void* x, int64_t ldx, const void* up, int64_t ldup, int dtype, int64_t rows, int64_t cols, int kind,
                             void* y, int64_t ldy, int8_t* x_codes, float* x_scales, int8_t* up_codes, float* up_scales, void* stream) {
  unsigned blocks;
  if (const int rc = check_rows(rows, cols, &blocks)) return rc;
  const bool gated = up != nullptr, keep = x_codes != nullptr || x_scales != nullptr;
  if (ldx < cols || ldy < cols || (gated && ldup < cols)) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (kind != EFQAT_ACT_GELU && kind != EFQAT_ACT_SILU) return EFQAT_ERR_BAD_LAYOUT;
  if (!x || !y) return EFQAT_ERR_NULL_PTR;
  if (keep && (!x_codes || !x_scales || (gated && (!up_codes || !up_scales)))) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(x, dtype) || !aligned_for(y, dtype) || !aligned_for(up, dtype)) return EFQAT_ERR_ALIGNMENT;
  if (keep && (!aligned16(x_codes) || !aligned4(x_scales) || (gated && (!aligned16(up_codes) || !aligned4(up_scales)))))
    return EFQAT_ERR_ALIGNMENT;
  const uint32_t gpr = (uint32_t)ckpt_groups(cols);
  const Ckpt kx = {x_codes, x_scales}, ku = {up_codes, up_scales};
  hipStream_t st = (hipStream_t)stream;
#define EFQAT_ACT(E, KIND, G, K) \
  EFQAT_TRY(launch((k_act_fwd<E, KIND, G, K>), dim3(blocks), dim3(256), 0, st, (const E*)x, ldx, (const E*)up, ldup, rows, cols, gpr, (E*)y, ldy, kx, ku))
#define EFQAT_ACT_K(E, G, K) do { if (kind == EFQAT_ACT_GELU) EFQAT_ACT(E, EFQAT_ACT_GELU, G, K); else EFQAT_ACT(E, EFQAT_ACT_SILU, G, K); } while (0)
#define EFQAT_ACT_G(E, K) do { if (gated) EFQAT_ACT_K(E, true, K); else EFQAT_ACT_K(E, false, K); } while (0)
  if (dtype == EFQAT_F32) { if (keep) EFQAT_ACT_G(float, true); else EFQAT_ACT_G(float, false); }
  else { if (keep) EFQAT_ACT_G(bf16_t, true); else EFQAT_ACT_G(bf16_t, false); }
#undef EFQAT_ACT_G
#undef EFQAT_ACT_K
#undef EFQAT_ACT
  return EFQAT_OK;
}

extern "C" int efqat_act_bwd(const void* dy, int64_t lddy, int dtype, int64_t rows, int64_t cols, int kind, const int8_t* x_codes,
                             const float* x_scales, const int8_t* up_codes, const float* up_scales, void* dx, int64_t lddx, void* dup,
                             int64_t lddup, void* stream) {
  unsigned blocks;
  if (const int rc = check_rows(rows, cols, &blocks)) return rc;
  const bool gated = up_codes != nullptr || up_scales != nullptr || dup != nullptr;
  if (lddy < cols || lddx < cols || (gated && lddup < cols)) return EFQAT_ERR_BAD_SHAPE;
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (kind != EFQAT_ACT_GELU && kind != EFQAT_ACT_SILU) return EFQAT_ERR_BAD_LAYOUT;
  if (!dy || !x_codes || !x_scales || !dx || (gated && (!up_codes || !up_scales || !dup))) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(dy, dtype) || !aligned_for(dx, dtype) || !aligned_for(dup, dtype) || !aligned16(x_codes) || !aligned4(x_scales) ||
      !aligned16(up_codes) || !aligned4(up_scales))
    return EFQAT_ERR_ALIGNMENT;
  const uint32_t gpr = (uint32_t)ckpt_groups(cols);
  const Ckpt kx = {const_cast<int8_t*>(x_codes), const_cast<float*>(x_scales)};
  const Ckpt ku = {const_cast<int8_t*>(up_codes), const_cast<float*>(up_scales)};
  hipStream_t st = (hipStream_t)stream;
#define EFQAT_ACT(E, KIND, G) \
  EFQAT_TRY(launch((k_act_bwd<E, KIND, G>), dim3(blocks), dim3(256), 0, st, (const E*)dy, lddy, rows, cols, gpr, kx, ku, (E*)dx, lddx, (E*)dup, lddup))
#define EFQAT_ACT_K(E, G) do { if (kind == EFQAT_ACT_GELU) EFQAT_ACT(E, EFQAT_ACT_GELU, G); else EFQAT_ACT(E, EFQAT_ACT_SILU, G); } while (0)
  if (dtype == EFQAT_F32) { if (gated) EFQAT_ACT_K(float, true); else EFQAT_ACT_K(float, false); }
  else { if (gated) EFQAT_ACT_K(bf16_t, true); else EFQAT_ACT_K(bf16_t, false); }
#undef EFQAT_ACT_K
#undef EFQAT_ACT
  return EFQAT_OK;
}
