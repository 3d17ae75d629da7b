// Rows of activations in chunks of 8 columns, and the 8-bit checkpoint of a row (see efqat_ckpt8_save), shared by the
// elementwise and the row-wise kernels.
#pragma once
#include "common.hpp"

#include <tuple>
#include <type_traits>

namespace efqat {

constexpr int kCkptGroup = EFQAT_CKPT8_GROUP;         // columns that share a scale
constexpr int kGroupLanes = kCkptGroup / 8;           // lanes of a group: 16, one DPP row

// 8 elements at p as they lie in memory, at any element alignment (the hardware takes vector accesses there)
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
  typedef float vec __attribute__((ext_vector_type(4), aligned(4)));
  vec a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const vec*>(p);
    b = *reinterpret_cast<const vec*>(p + 4);
  }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
  }
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[i] = v[i]; b[i] = v[4 + i]; }
  }
  __device__ __forceinline__ void store(float* p) const {
    *reinterpret_cast<vec*>(p) = a;
    *reinterpret_cast<vec*>(p + 4) = b;
  }
};
template <>
struct Raw8<bf16_t> {
  typedef uint32_t vec __attribute__((ext_vector_type(4), aligned(2)));
  vec a;
  __device__ __forceinline__ void load(const bf16_t* p) { a = *reinterpret_cast<const vec*>(p); }
  __device__ __forceinline__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(a[i] << 16);
      v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
    }
  }
  // rounded to nearest even, infinities and NaN kept
  __device__ __forceinline__ void set(const float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
  }
  __device__ __forceinline__ void store(bf16_t* p) const { *reinterpret_cast<vec*>(p) = a; }
};

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ bf16_t from_f32<bf16_t>(float v) { return (bf16_t)(pack_bf16x2(v, v) & 0xFFFFu); }

// The chunk of the n <= 8 first elements at p (n <= 0: none); what lies behind them is neither read nor written.
template <typename T>
__device__ __forceinline__ Raw8<T> load_chunk(const T* p, int n) {
  Raw8<T> r;
  if (n >= 8) {
    r.load(p);
  } else {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = j < n ? load_as_f32<T>(p, j) : 0.0f;
    r.set(v);                                         // bf16 values come through unchanged (a NaN stays one)
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* p, int n, const float (&v)[8]) {
  if (n >= 8) {
    Raw8<T> r;
    r.set(v);
    r.store(p);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = from_f32<T>(v[j]);
  }
}

// Place of a chunk in rows of cols >= 8 elements that are read without a branch: a chunk that passes the end is the row's last 8
// elements, moved down by `shift` with zeros behind them; one that begins behind the end (shift 8) is zeros.
struct ChunkPlace {
  int at, shift, n;               // first element that is read; elements to move; elements that exist
  __device__ __forceinline__ ChunkPlace() {}
  __device__ __forceinline__ ChunkPlace(int64_t cols, int64_t col) {
    const int64_t over = col + 8 - cols;
    at = (int)(over > 0 ? cols - 8 : col);
    shift = (int)(over < 0 ? 0 : over > 8 ? 8 : over);
    n = 8 - shift;
  }
};
// element j + shift in the place of element j, shift < 8
__device__ __forceinline__ void move_down(float (&v)[8], int shift) {
#pragma unroll
  for (int s = 4; s > 0; s >>= 1)
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = shift & s ? (j + s < 8 ? v[j + s < 8 ? j + s : 7] : 0.0f) : v[j];
}
template <typename T>
__device__ __forceinline__ void get_chunk(const Raw8<T>& r, const ChunkPlace& c, float (&v)[8]) {
  r.get(v);
  if (c.shift >= 8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = 0.0f;
  } else if (c.shift > 0) {
    move_down(v, c.shift);
  }
}

// ---- the 8-bit checkpoint: bytes a row of codes takes, scales a row has
__host__ __device__ inline int64_t ckpt_pitch(int64_t cols) { return round_up(cols, 16); }
__host__ __device__ inline int64_t ckpt_groups(int64_t cols) { return ceil_div(cols, kCkptGroup); }

// the largest of the 16 lanes of a DPP row, in all of them
__device__ __forceinline__ uint32_t group_max(uint32_t v) {
  auto step = [&](uint32_t o) { v = v > o ? v : o; };
  step(__builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, true));      // quad_perm: lane ^ 1
  step(__builtin_amdgcn_update_dpp(0, v, 0x4E, 0xF, 0xF, true));      // quad_perm: lane ^ 2
  step(__builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, true));     // row_half_mirror: lane -> 7 - lane
  step(__builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, true));     // row_mirror: lane -> 15 - lane
  return v;
}

// the sum of a wavefront, in all its lanes: rows of 16 by DPP, the four rows through scalar registers, in a fixed order (a butterfly
// over __shfl_xor goes through LDS six times)
__device__ __forceinline__ float wave_total(float v) {
  auto add = [&](int o) { v += __builtin_bit_cast(float, o); };
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x141, 0xF, 0xF, true));
  add(__builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x140, 0xF, 0xF, true));
  auto row = [&](int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); };
  return (row(0) + row(16)) + (row(32) + row(48));
}

// Codes of a chunk and the scale of its group; all 16 lanes of the group take part (chunks without columns hold zeros).
// scale = max(max|x| fl(1/127), 2^-126), code = rne(x fl(1/scale)), in fp32: |x| (1/scale) is at most 127 (1 + 2^-22).  The
// magnitudes are compared as integers, where a NaN is larger than everything: a group that holds an infinity or a NaN has a
// NaN for its scale, and all of it reads back as that.
__device__ __forceinline__ uint2 ckpt_encode(const float (&v)[8], float* scale) {
  uint32_t m = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t a = __float_as_uint(v[j]) & 0x7FFFFFFFu;
    m = m > a ? m : a;
  }
  float s = __uint_as_float(group_max(m)) * (1.0f / 127.0f);
  s = s < INFINITY ? s : NAN;
  s = s < 0x1p-126f ? 0x1p-126f : s;
  *scale = s;
  const float inv = 1.0f / s;
  // the product is rounded first, then to an integer by the addition: the lowest byte of 1.5 2^23 + q is q in two's complement
  uint32_t t[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) t[j] = __float_as_uint(__fadd_rn(__fmul_rn(v[j], inv), 12582912.0f));
  auto four = [&](int j) {                            // the lowest bytes of four words
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[j + 3], t[j + 2], 0x0C0C0400u), __builtin_amdgcn_perm(t[j + 1], t[j], 0x0C0C0400u),
                                 0x05040100u);
  };
  return make_uint2(four(0), four(4));
}
// code * scale, rounded once.  The product is formed from the signed code: 128 * scale may be infinite where 127 * scale, the largest
// kept value, is not.  A byte's sign is extended by the conversion itself.
__device__ __forceinline__ void ckpt_decode(uint2 codes, float scale, float (&v)[8]) {
  const uint32_t w[2] = {codes.x, codes.y};
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(w[j >> 2] >> (8 * (j & 3))) * scale;
}

// Launches a kernel and says whether that went well by what the launch itself returns: the last error of the thread may be one
// that another library left there (and is left for it).
template <class... P, class... A>
inline int launch(void (*kernel)(P...), dim3 grid, dim3 block, size_t lds, hipStream_t st, const A&... a) {
  std::tuple<std::remove_cv_t<P>...> args{static_cast<std::remove_cv_t<P>>(a)...};
  return std::apply(
      [&](auto&... x) {
        void* at[] = {(void*)&x...};
        return hipLaunchKernel((const void*)kernel, grid, block, at, lds, st) == hipSuccess ? EFQAT_OK : EFQAT_ERR_HIP;
      },
      args);
}

#define EFQAT_TRY(...)                         \
  do {                                         \
    if (const int rc_ = (__VA_ARGS__)) return rc_; \
  } while (0)

inline bool known_dtype(int dtype) { return dtype == EFQAT_F32 || dtype == EFQAT_BF16; }
inline bool aligned_for(const void* p, int dtype) { return ((uintptr_t)p % (dtype == EFQAT_F32 ? 4 : 2)) == 0; }
inline bool aligned16(const void* p) { return ((uintptr_t)p % 16) == 0; }
inline bool aligned4(const void* p) { return ((uintptr_t)p % 4) == 0; }

}  // namespace efqat
