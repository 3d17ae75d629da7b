// Dropout whose mask is drawn from a counter and never stored:
//
//   y = [residual +] [u >= t] x 65536 / (65536 - t),  t = rne(65536 p)
//
// u is 16 bits of Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011): chunk n of 8 columns,
// counted along the rows, takes the four words of the counter (n, offset) under the key seed, the lower half of a word first.  The mask is
// thus a function of seed, offset and an element's place alone: the backward pass draws it again, and neither strides nor types change it.
//
// Bound by HBM: one pass, 16 bytes (bf16) or 32 a lane and tensor; the ten rounds are 20 wide multiplications for 8 elements.
// bf16, 12288 x 768 with residual: 11 us (57 MB, 5.0 TB/s); fp32, 2049 x 1001: 4.8 us, a launch.
#include "rows.hpp"

namespace efqat {

__device__ __forceinline__ uint4 philox(uint4 c, uint2 k) {
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t a = (uint64_t)c.x * 0xD2511F53u, b = (uint64_t)c.z * 0xCD9E8D57u;
    c = make_uint4((uint32_t)(b >> 32) ^ c.y ^ k.x, (uint32_t)b, (uint32_t)(a >> 32) ^ c.w ^ k.y, (uint32_t)a);
    k.x += 0x9E3779B9u;
    k.y += 0xBB67AE85u;
  }
  return c;
}

constexpr int64_t kDropoutBlocks = 1 << 23;           // a grid has fewer than 2^32 lanes

template <typename T, bool RESIDUAL>
__global__ __launch_bounds__(256) void k_dropout(const T* x, int64_t ldx, const T* res, int64_t ldr, int64_t rows, int64_t cols, uint32_t cpr,
                                                 uint32_t least, float scale, const int64_t* __restrict__ state, T* y, int64_t ldy) {
  // 256 chunks a block and step, numbered along the rows
  for (uint64_t first = (uint64_t)blockIdx.x * 256; first < (uint64_t)rows * cpr; first += (uint64_t)gridDim.x * 256) {
    const uint64_t row0 = first / cpr;
    const uint32_t at = (uint32_t)(first - row0 * cpr) + threadIdx.x;       // cpr < 2^29
    const uint32_t more = at / cpr;
    const int64_t row = (int64_t)row0 + more, col = (int64_t)(at - more * cpr) * 8;
    if (row >= rows) return;                         // the last step
    const int64_t left = cols - col;
    const int n = left > 8 ? 8 : (int)left;
    const Raw8<T> rx = load_chunk(x + row * ldx + col, n);
    Raw8<T> rr;
    if constexpr (RESIDUAL) rr = load_chunk(res + row * ldr + col, n);
    const uint64_t seed = (uint64_t)state[0], offset = (uint64_t)state[1], chunk = first + threadIdx.x;
    const uint4 u = philox(make_uint4((uint32_t)chunk, (uint32_t)(chunk >> 32), (uint32_t)offset, (uint32_t)(offset >> 32)),
                           make_uint2((uint32_t)seed, (uint32_t)(seed >> 32)));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    float v[8], b[8];
    rx.get(v);
    if constexpr (RESIDUAL) rr.get(b);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t bits = j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu;
      const float kept = RESIDUAL ? fmaf(v[j], scale, b[j]) : v[j] * scale;
      v[j] = bits >= least ? kept : RESIDUAL ? b[j] : 0.0f;          // chosen, not multiplied: a dropped infinity or NaN leaves nothing behind
    }
    store_chunk(y + row * ldy + col, n, v);
  }
}

}  // namespace efqat

using namespace efqat;

extern "C" int efqat_dropout(const void* x, int64_t ldx, const void* residual, int64_t ldr, int dtype, int64_t rows, int64_t cols, double p,
                             const int64_t* state, void* y, int64_t ldy, void* stream) {
  if (rows <= 0 || cols <= 0 || rows > INT64_C(1) << 34 || cols > INT32_MAX || ldx < cols || ldy < cols || (residual && ldr < cols) ||
      !(p >= 0.0) || !(p <= 1.0))
    return EFQAT_ERR_BAD_SHAPE;
  const int64_t cpr = ceil_div(cols, 8);
  if (!known_dtype(dtype)) return EFQAT_ERR_BAD_DTYPE;
  if (!x || !y || !state) return EFQAT_ERR_NULL_PTR;
  if (!aligned_for(x, dtype) || !aligned_for(y, dtype) || !aligned_for(residual, dtype) || (uintptr_t)state % 8) return EFQAT_ERR_ALIGNMENT;
  const uint32_t least = (uint32_t)__builtin_rint(p * 65536.0);
  const float scale = least < 65536 ? 65536.0f / (float)(65536 - least) : 0.0f;
  const int64_t blocks = ceil_div(rows * cpr, 256);
  const dim3 grid((unsigned)(blocks < kDropoutBlocks ? blocks : kDropoutBlocks));
  hipStream_t st = (hipStream_t)stream;
#define EFQAT_DROP(E, R)                                                                                                      \
  return launch(k_dropout<E, R>, grid, dim3(256), 0, st, (const E*)x, ldx, (const E*)residual, ldr, rows, cols, (uint32_t)cpr, least, scale, \
                state, (E*)y, ldy)
  if (dtype == EFQAT_F32) { if (residual) EFQAT_DROP(float, true); EFQAT_DROP(float, false); }
  if (residual) EFQAT_DROP(bf16_t, true);
  EFQAT_DROP(bf16_t, false);
#undef EFQAT_DROP
}
