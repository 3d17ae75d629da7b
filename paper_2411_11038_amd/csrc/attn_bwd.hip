// Backward of attention with a sliding window and first tokens that stay visible (see attn.hip), from lse and without kept scores:
//
//   P_ij = exp(scale q_i . k_j - lse_i) over the keys that token i sees,  dP_ij = do_i . v_j,  delta_i = do_i . o_i,
//   dS_ij = P_ij (dP_ij - delta_i),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij do_i
//
// Two kernels, each with the sums of its outputs in registers: k_attn_dq walks the keys of 128 queries, k_attn_dkv the queries (of all
// heads that share them) of 128 keys.  Scores and dP are formed twice, seven products instead of the five that one kernel would need, but
// no sum crosses blocks: nothing is added by atomics, and results do not change from run to run.  With bf16 operands P and dS are
// rounded to bf16 for the matrix cores, as probabilities are in the forward pass.
#include "attn_tile.hpp"

namespace efqat {

constexpr float kLog2e = 1.4426950408889634f;

struct AttnGrads {
  const void *dout, *o;
  int64_t lddo, ldo;
  const float* lse;                                  // [heads][rows]
  float* delta;                                      // [heads][rows]
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
};

// What prob() takes of a token's lse, and the factor of the scores.  bf16: exp2(s c - lse log2 e), one operation beside the exponential.
// fp32: exp2((s scale - lse) log2 e), whose argument is small wherever the result is not, and exact to 2^-24 of it.
template <typename T>
__device__ __forceinline__ float prob_base(float lse) {
  return lse == -INFINITY ? INFINITY : sizeof(T) == 2 ? lse * kLog2e : lse;       // a token that sees nothing: P = 0
}
template <typename T>
__device__ __forceinline__ float prob(float s, float c, float base) {
  const float x = fmaf(s, c, -base);
  return __builtin_amdgcn_exp2f(sizeof(T) == 2 ? x : x * kLog2e);
}
template <typename T>
__device__ __forceinline__ float prob_factor(float scale) { return sizeof(T) == 2 ? scale * kLog2e : scale; }

// dq, and delta for the other kernel.  Blocks and layout as in k_attn_fwd.
template <typename T, int DP, int NW>
__global__ __launch_bounds__(64 * NW, (kWideBlocks<T, DP> ? 2 : 1)) void k_attn_dq(AttnArgs a, AttnGrads g, int tiles, int hb) {
  using R = RowTile<T, DP>;
  constexpr int BN = kKeyStage<T>, STAGE = 2 * BN * R::ROW;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  HeadTile w;
  if (!w.find(a, NW, hb, tiles, wave)) return;
  const int p = w.row + (lane & 31) + w.shift, head = w.head;
  const KeyTiles kt(a.mask, w.keys.y, w.block_row + w.shift, w.block_row + w.block_rows - 1 + w.shift, BN);
  KeyCopies<T, DP, NW> copies(a, w.keys, w.kvh, wave);
  if (kt.count > 0) copies.issue(kt.tile(0), smem, wave);

  const bool in = w.in(lane);
  const int64_t row = w.token(lane);
  Frag<T> q[R::KS], d[R::KS];
  float delta = 0.0f, lse = INFINITY;
  {
    const T* qr = (const T*)a.q + row * a.ldq + head * a.dim;
    const T* dr = (const T*)g.dout + row * g.lddo + head * a.dim;
    const T* orow = (const T*)g.o + row * g.ldo + head * a.dim;
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks) {
      const int c = 16 * ks + 8 * (lane >> 5);
      const bool ok = in && c < a.dim;
      q[ks] = load_frag(qr + c, ok);
      d[ks] = load_frag(dr + c, ok);
      const Frag<T> of = load_frag(orow + c, ok);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)d[ks].v[e], (float)of.v[e], delta);
    }
    delta = half_sum(delta);
    if (in) {
      lse = prob_base<T>(g.lse[(int64_t)head * a.qs.rows + row]);
      if (lane < 32) g.delta[(int64_t)head * a.qs.rows + row] = delta;
    }
  }
  floatx16_t acc[R::ND];
#pragma unroll
  for (int i = 0; i < R::ND; ++i) acc[i] = zero16();
  const float c = prob_factor<T>(a.scale);
  tile_sync();
  for (int t = 0; t < kt.count; ++t) {
    char* buf = smem + (t & 1) * STAGE;
    if (t + 1 < kt.count) copies.issue(kt.tile(t + 1), smem + ((t + 1) & 1) * STAGE, wave);
    const int p0 = w.row + w.shift, p1 = p0 + 31;
#pragma unroll
    for (int n = 0; n < BN / 32; ++n) {
      const int j0 = kt.tile(t) * BN + 32 * n;
      auto tile = [&](auto masked) {
        floatx16_t s = zero16(), dp = zero16();
#pragma unroll
        for (int ks = 0; ks < R::KS; ++ks) {
          mma(R::row_frag(buf, 32 * n, ks), q[ks], s);
          mma(R::row_frag(buf + BN * R::ROW, 32 * n, ks), d[ks], dp);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[i] = prob<T>(s[i], c, lse) * (dp[i] - delta);
          if constexpr (decltype(masked)::value) {
            const int j = j0 + result_row(i);
            s[i] = ((j < w.keys.y) & a.mask.sees(p, j)) ? s[i] : 0.0f;
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Frag<T> f = frag_of<T>(s, h);
#pragma unroll
          for (int i = 0; i < R::ND; ++i) mma(R::col_frag(buf, 32 * n + 16 * h, i), f, acc[i]);
        }
      };
      if (a.mask.sees_some(p0, p1, j0, j0 + 31)) {
        if (j0 + 32 <= w.keys.y && a.mask.sees_all(p0, p1, j0, j0 + 31)) tile(std::false_type{});
        else tile(std::true_type{});
      }
    }
    tile_sync();
  }
  results_settle();
  store_rows<T, DP>((T*)g.dq + w.token(0) * g.lddq + head * a.dim, g.lddq, w.rows_left(), a.dim, acc, a.scale, smem + wave * (sizeof(smem) / NW));
}

// Queries first .. last - 1 of a sequence that see some of the keys j0 .. j1
struct QuerySpan {
  int first, last;
  __device__ __forceinline__ QuerySpan(const AttnMask& m, int queries, int shift, int j0, int j1) {
    int lo = m.causal ? j0 - shift : 0, hi = queries;
    if (m.window && j0 >= m.sinks) {
      const int past = j1 + m.window - shift, before = j0 - m.window + 1 - shift;
      hi = past < hi ? past : hi;
      lo = before > lo ? before : lo;
    }
    first = lo < 0 ? 0 : lo;
    last = hi;
  }
};

// dk and dv of 128 keys, 32 a wavefront: scores with queries as rows and keys as columns, so that P and dS are operands of the sums over
// the queries where they are.
template <typename T, int DP>
__global__ __launch_bounds__(256, 1) void k_attn_dkv(AttnArgs a, AttnGrads g, int tiles) {
  using R = RowTile<T, DP>;
  constexpr int BM = 128, BQ = sizeof(T) == 2 ? 64 : 32, STAGE = 2 * BQ * R::ROW;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE];
  __shared__ __attribute__((aligned(16))) float s_lse[2][BQ], s_delta[2][BQ];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int id = xcd_contiguous_index(blockIdx.x, gridDim.x);
  const int kvh = id / tiles;
  int seq, tile;
  if (!find_tile(a.ks, BM, id - kvh * tiles, &seq, &tile)) return;
  const int2 qp = a.qs.place(seq), kp = a.ks.place(seq);
  const int shift = kp.y - qp.y, k0 = tile * BM + wave * 32, krow = k0 + (lane & 31);
  const QuerySpan span(a.mask, qp.y, shift, tile * BM, min(tile * BM + BM, kp.y) - 1);
  const int nq = span.last > span.first ? (span.last - span.first + BQ - 1) / BQ : 0, count = nq * a.group;

  const int64_t ldq = a.ldq * (int)sizeof(T), lddo = g.lddo * (int)sizeof(T);
  const int pieces = a.dim * (int)sizeof(T) / 16;
  float next_lse = 0.0f, next_delta = 0.0f;
  auto issue = [&](int t, char* buf) {
    const int head = kvh * a.group + t / nq, i0 = span.first + (t % nq) * BQ, valid = qp.y - i0;
    const char* qbase = (const char*)((const T*)a.q + (int64_t)(qp.x + i0) * a.ldq + head * a.dim);
    const char* dbase = (const char*)((const T*)g.dout + (int64_t)(qp.x + i0) * g.lddo + head * a.dim);
#pragma unroll
    for (int s = 0; s < BQ / R::RPI / 4; ++s) R::copy(qbase, ldq, valid, pieces, buf, wave + 4 * s);
#pragma unroll
    for (int s = 0; s < BQ / R::RPI / 4; ++s) R::copy(dbase, lddo, valid, pieces, buf + BQ * R::ROW, wave + 4 * s);
    if (threadIdx.x < BQ) {
      const int i = threadIdx.x;
      const int64_t from = (int64_t)head * a.qs.rows + qp.x + i0 + i;
      next_lse = INFINITY;                                          // rows behind the sequence and tokens that see nothing: P = 0
      next_delta = 0.0f;
      if (i < valid) {
        next_lse = prob_base<T>(g.lse[from]);
        next_delta = g.delta[from];
      }
    }
  };
  auto keep = [&](int b) {
    if (threadIdx.x < BQ) {
      s_lse[b][threadIdx.x] = next_lse;
      s_delta[b][threadIdx.x] = next_delta;
    }
  };
  if (count > 0) {
    issue(0, smem);
    keep(0);
  }

  const bool in = krow < kp.y;
  const int64_t row = (int64_t)kp.x + krow;
  Frag<T> k[R::KS], v[R::KS];
#pragma unroll
  for (int ks = 0; ks < R::KS; ++ks) {
    const int c = 16 * ks + 8 * (lane >> 5);
    k[ks] = load_frag((const T*)a.k + row * a.ldk + kvh * a.dim + c, in && c < a.dim);
    v[ks] = load_frag((const T*)a.v + row * a.ldv + kvh * a.dim + c, in && c < a.dim);
  }
  floatx16_t dk[R::ND], dv[R::ND];
#pragma unroll
  for (int i = 0; i < R::ND; ++i) dk[i] = dv[i] = zero16();
  const float c = prob_factor<T>(a.scale);
  tile_sync();
  for (int t = 0; t < count; ++t) {
    const int b = t & 1;
    char* buf = smem + b * STAGE;
    if (t + 1 < count) issue(t + 1, smem + (b ^ 1) * STAGE);
    const int i0 = span.first + (t % nq) * BQ;
#pragma unroll
    for (int n = 0; n < BQ / 32; ++n) {
      const int p0 = i0 + 32 * n + shift, p1 = p0 + 31;
      auto tile = [&](auto masked) {
        floatx16_t s = zero16(), dp = zero16();
#pragma unroll
        for (int ks = 0; ks < R::KS; ++ks) {
          mma(R::row_frag(buf, 32 * n, ks), k[ks], s);
          mma(R::row_frag(buf + BQ * R::ROW, 32 * n, ks), v[ks], dp);
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 l4 = *(const float4*)&s_lse[b][32 * n + result_row(i)];
          const float4 d4 = *(const float4*)&s_delta[b][32 * n + result_row(i)];
          const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, ds[4] = {d4.x, d4.y, d4.z, d4.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float e = prob<T>(s[i + j], c, ls[j]), f = e * (dp[i + j] - ds[j]);
            if constexpr (decltype(masked)::value) {
              const bool seen = a.mask.sees(p0 + result_row(i + j), krow);
              s[i + j] = seen ? e : 0.0f;
              dp[i + j] = seen ? f : 0.0f;
            } else {
              s[i + j] = e;
              dp[i + j] = f;
            }
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Frag<T> pf = frag_of<T>(s, h), df = frag_of<T>(dp, h);
#pragma unroll
          for (int i = 0; i < R::ND; ++i) {
            mma(R::col_frag(buf + BQ * R::ROW, 32 * n + 16 * h, i), pf, dv[i]);
            mma(R::col_frag(buf, 32 * n + 16 * h, i), df, dk[i]);
          }
        }
      };
      if (i0 + 32 * n < qp.y && a.mask.sees_some(p0, p1, k0, k0 + 31)) {
        if (a.mask.sees_all(p0, p1, k0, k0 + 31)) tile(std::false_type{});
        else tile(std::true_type{});
      }
    }
    if (t + 1 < count) keep(b ^ 1);
    tile_sync();
  }
  results_settle();
  if (in) {
    T* tk = (T*)g.dk + row * g.lddk + kvh * a.dim;
    T* tv = (T*)g.dv + row * g.lddv + kvh * a.dim;
#pragma unroll
    for (int i = 0; i < R::ND; ++i) {
      store_col(tk, dk[i], i, a.dim, a.scale);
      store_col(tv, dv[i], i, a.dim, 1.0f);
    }
  }
}

}  // namespace efqat

using namespace efqat;

extern "C" size_t efqat_attention_bwd_workspace_bytes(int64_t Tq, int64_t heads) {
  if (Tq <= 0 || heads <= 0 || Tq > kAttnMostRows || heads > 65535) return 256;
  return (size_t)round_up(Tq * heads * 4, 256);
}

extern "C" int efqat_attention_bwd(const void* dout, int64_t lddo, const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v,
                                   int64_t ldv, const void* o, int64_t ldo, const float* lse, int dtype, int64_t Tq, int64_t Tk, int64_t n_seq,
                                   const int32_t* q_start, const int32_t* k_start, int64_t heads, int64_t kv_heads, int64_t dim, float scale,
                                   int causal, int64_t window, int64_t sinks, void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv,
                                   int64_t lddv, void* ws, size_t ws_bytes, void* stream) {
  AttnArgs a;
  EFQAT_TRY(attn_args(&a, q, ldq, k, ldk, v, ldv, dtype, Tq, Tk, n_seq, q_start, k_start, heads, kv_heads, dim, scale, causal, window, sinks));
  EFQAT_TRY(attn_rows(dout, lddo, heads * dim, dtype));
  EFQAT_TRY(attn_rows(o, ldo, heads * dim, dtype));
  EFQAT_TRY(attn_rows(dq, lddq, heads * dim, dtype));
  EFQAT_TRY(attn_rows(dk, lddk, kv_heads * dim, dtype));
  EFQAT_TRY(attn_rows(dv, lddv, kv_heads * dim, dtype));
  if (!lse || !ws) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(lse) || (uintptr_t)ws % 256) return EFQAT_ERR_ALIGNMENT;
  if (ws_bytes < efqat_attention_bwd_workspace_bytes(Tq, heads)) return EFQAT_ERR_WORKSPACE;
  const HeadPlan h = head_plan(a, kv_heads, dtype);
  const int64_t kt = a.ks.most_tiles(128);
  if (h.blocks > kAttnMostBlocks || kt * kv_heads > kAttnMostBlocks) return EFQAT_ERR_BAD_SHAPE;
  const AttnGrads g = {dout, o, lddo, ldo, lse, (float*)ws, dq, dk, dv, lddq, lddk, lddv};
  hipStream_t st = (hipStream_t)stream;
#define EFQAT_BWD(E, DP)                                                                                             \
  do {                                                                                                               \
    if (h.waves == 8) {                                                                                              \
      if constexpr (kWideBlocks<E, DP>) EFQAT_TRY(launch(k_attn_dq<E, DP, 8>, dim3((unsigned)h.blocks), dim3(512), 0, st, a, g, h.tiles, h.hb)); \
    } else EFQAT_TRY(launch(k_attn_dq<E, DP, 4>, dim3((unsigned)h.blocks), dim3(256), 0, st, a, g, h.tiles, h.hb));    \
    return launch(k_attn_dkv<E, DP>, dim3((unsigned)(kt * kv_heads)), dim3(256), 0, st, a, g, (int)kt);              \
  } while (0)
  if (dtype == EFQAT_F32) { if (dim <= 64) EFQAT_BWD(float, 64); EFQAT_BWD(float, 128); }
  if (dim <= 64) EFQAT_BWD(bf16_t, 64);
  EFQAT_BWD(bf16_t, 128);
#undef EFQAT_BWD
}
