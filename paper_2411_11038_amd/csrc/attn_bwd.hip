// Backward of attention with a sliding window and first tokens that stay visible (see attn.hip), from lse and without kept scores:
//
//   P_ij = exp(scale q_i . k_j - lse_i) over the keys that token i sees,  dP_ij = do_i . v_j,  delta_i = do_i . o_i,
//   dS_ij = P_ij (dP_ij - delta_i),  dq_i = scale sum_j dS_ij k_j,  dk_j = scale sum_i dS_ij q_i,  dv_j = sum_i P_ij do_i
//
// Two kernels, each with the sums of its outputs in registers: k_attn_dq walks the keys of 128 queries, k_attn_dkv the queries (of all
// heads that share them) of 128 keys.  Scores and dP are formed twice: seven products with fp32 (three and four) instead of the five that one
// kernel would need, nine with bf16, whose dq takes two more (below).  But no sum crosses blocks: nothing is added by atomics, and results do
// not change from run to run.  With bf16 operands P and, for dk, dS are
// rounded to bf16 for the matrix cores, as probabilities are in the forward pass; dq takes dS as two such parts.
//
// Bound by the matrix cores and what is issued beside them.  2 x 4096 tokens, 32 query and 8 key heads of 128, window 1024, 4 sinks: dq 320 us (0.94 PFLOP/s
// in five products), dk and dv 414 us (0.58 in four; 256 of their 776 blocks are the sinks' far parts), 9 us to join them.  32 x 384 tokens, 12 heads
// of 64: 64 and 66 us, six stages a block.  fp32, 7 sequences, 3001 tokens in all, heads of 80: 124 and 156 us and 10 to join, the rate of fp32
// matrix instructions on the longest blocks.  (Kernel times of a trace, medians; a launch's start and end are in each.)
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

// dq, and delta for the other kernel.  Blocks as in k_attn_fwd.  (Forming the next 32 keys' scores beside dS, as k_attn_fwd does, needs
// more registers than two wavefronts a SIMD have: 380 instead of 250 us for a window of 1024 in 2 x 4096 tokens, 32 heads of 128.)
//
// bf16: o is rounded, and delta from it is off by up to 2^-8 of do . o, far more than dS where one key takes nearly all of P (dq 0.5 % off in the
// 2-norm for short sequences; the mend took dq of a window of 1024 from 254 to 300 us, the second part of dS from 290 to 323).  Exactly, sum_j dS_ij = 0: what it comes to is what delta lacks, d_i.  So sum_j P_ij k_j is formed too, from the
// fragments of k that are there, and  dq_i = scale (sum_j dS_ij k_j - d_i sum_j P_ij k_j).  d is small: P need not be exact there.
template <typename T, int DP>
struct DqTile {
  static constexpr bool MEND = sizeof(T) == 2, QUERIES_IN_LDS = MEND && DP == 128;         // the second sum takes the queries' registers
  static constexpr int BN = QUERIES_IN_LDS ? 32 : kKeyStage<T>;
};
template <typename T, int DP>
__global__ __launch_bounds__(256, (kTwoWaves<T, DP> ? 2 : 1)) void k_attn_dq(AttnArgs a, AttnGrads g, int tiles, int hb) {
  using R = RowTile<T, DP>;
  using C = DqTile<T, DP>;
  constexpr int BN = C::BN, STAGE = 2 * BN * R::ROW, OWN = 32 * R::ROW;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE + (C::QUERIES_IN_LDS ? 4 * OWN : 0)];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  HeadTile w;
  if (!w.find(a, hb, tiles, wave)) return;
  const int p = w.row + (lane & 31) + w.shift, head = w.head;
  const KeyTiles kt(a.mask, w.keys.y, w.block_row + w.shift, w.block_row + w.block_rows - 1 + w.shift, BN);
  KeyCopies<T, DP, BN> copies(a, w.keys, w.kvh, wave);
  char* const own = smem + 2 * STAGE + wave * OWN;
  if constexpr (C::QUERIES_IN_LDS) {
#pragma unroll
    for (int s = 0; s < 32 / R::RPI; ++s)
      R::copy((const char*)((const T*)a.q + w.token(0) * a.ldq + head * a.dim), a.ldq * (int)sizeof(T), w.rows_left(),
              a.dim * (int)sizeof(T) / 16, own, s);
  }
  if (kt.count > 0) copies.issue(kt.tile(0), smem, wave);

  const bool in = w.in(lane);
  const int64_t row = w.token(lane);
  Frag<T> q[C::QUERIES_IN_LDS ? 1 : R::KS], d[R::KS];
  float delta = 0.0f, lse = prob_base<T>(-INFINITY), lack = 0.0f;
  {
    const T* qr = (const T*)a.q + row * a.ldq + head * a.dim;
    const T* dr = (const T*)g.dout + row * g.lddo + head * a.dim;
    const T* orow = (const T*)g.o + row * g.ldo + head * a.dim;
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks) {
      const int c = 16 * ks + 8 * (lane >> 5);
      const bool ok = in && c < a.dim;
      if constexpr (!C::QUERIES_IN_LDS) q[ks] = load_frag(qr + c, ok);
      d[ks] = load_frag(dr + c, ok);
      const Frag<T> of = load_frag(orow + c, ok);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)d[ks].v[e], (float)of.v[e], delta);
    }
    delta = half_sum(delta);
    if (in) lse = prob_base<T>(g.lse[(int64_t)head * a.qs.rows + row]);
  }
  floatx16_t acc[R::ND], mean[C::MEND ? R::ND : 1];
#pragma unroll
  for (int i = 0; i < R::ND; ++i) {
    acc[i] = zero16();
    if constexpr (C::MEND) mean[i] = zero16();
  }
  const float c = prob_factor<T>(a.scale);
  tile_sync();
  for (int t = 0; t < kt.count; ++t) {
    char* buf = smem + (t & 1) * STAGE;
    if (t + 1 < kt.count) copies.issue(kt.tile(t + 1), smem + ((t + 1) & 1) * STAGE, wave);
    const int p0 = w.row + w.shift, p1 = p0 + 31;
#pragma unroll
    for (int n = 0; n < BN / 32; ++n) {
      const int j0 = kt.tile(t) * BN + 32 * n;
      if (!a.mask.sees_some(p0, p1, j0, j0 + 31)) continue;
      floatx16_t s = zero16(), dp = zero16();
#pragma unroll
      for (int ks = 0; ks < R::KS; ++ks) {
        if constexpr (C::QUERIES_IN_LDS) mma(R::row_frag(buf, 32 * n, ks), R::row_frag(own, 0, ks), s);
        else mma(R::row_frag(buf, 32 * n, ks), q[ks], s);
        mma(R::row_frag(buf + BN * R::ROW, 32 * n, ks), d[ks], dp);
      }
      results_settle();
      if (j0 + 32 > w.keys.y || !a.mask.sees_all(p0, p1, j0, j0 + 31)) {
        const int first = j0 + row_here();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int j = first + row_of(i);
          s[i] = ((j < w.keys.y) & a.mask.sees(p, j)) ? s[i] : -INFINITY;
        }
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = prob<T>(s[i], c, lse);
        dp[i] = s[i] * (dp[i] - delta);
      }
      if constexpr (C::MEND) lack += sum16(dp);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Frag<T> df = frag_of<T>(dp, h);
        Frag<T> pf, rest;
        if constexpr (C::MEND) {
          pf = frag_of<T>(s, h);
          rest = rest_of(dp, h, df);
        }
#pragma unroll
        for (int i = 0; i < R::ND; ++i) {
          const Frag<T> kf = R::col_frag(buf, 32 * n + 16 * h, i);
          mma(kf, df, acc[i]);
          if constexpr (C::MEND) {
            mma(kf, pf, mean[i]);
            mma(kf, rest, acc[i]);
          }
        }
      }
    }
    tile_sync();
  }
  results_settle();
  if constexpr (C::MEND) {
    lack = half_sum(lack);
#pragma unroll
    for (int i = 0; i < R::ND; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = fmaf(-lack, mean[i][r], acc[i][r]);
  }
  if (in && lane < 32) g.delta[(int64_t)head * a.qs.rows + row] = delta + lack;
  store_rows<T, DP>((T*)g.dq + w.token(0) * g.lddq + head * a.dim, g.lddq, w.rows_left(), a.dim, acc, a.scale, smem + wave * (sizeof(smem) / kWaves));
}

// Queries first .. last - 1 of a sequence that see some of the keys j0 .. j1; near: those that do beside what sinks add
struct QuerySpan {
  int first, last;
  __device__ __forceinline__ QuerySpan(const AttnMask& m, bool near, int queries, int shift, int j0, int j1) {
    int lo = m.causal ? j0 - shift : 0, hi = queries;
    if (m.window && (near || j0 >= m.sinks)) {
      const int past = j1 + m.window - shift, before = j0 - m.window + 1 - shift;
      hi = past < hi ? past : hi;
      lo = before > lo ? before : lo;
    }
    first = lo < 0 ? 0 : lo;
    last = hi;
  }
};

// How the work of dk and dv is cut.  `parts` blocks share a tile of 128 keys where there are few tiles.  Keys that stay visible beside a window
// have the queries of the whole sequence behind them, which one block would walk long after the others have ended: what lies outside their
// window is the work of `far` blocks of its own.  Parts leave fp32 sums in the workspace, which k_attn_dkv_join adds in their order.
struct KeyPlan {
  int tiles, parts, far, sink_tiles;
  int64_t near_blocks, far_blocks, slots;            // slots: sums of a block in the workspace
};
constexpr int kKeyRows = 128;
// sums of a block of (tile, head) and part; far parts and, where tiles are not cut, the near part of a tile with sinks lie behind them
__host__ __device__ inline int64_t near_slot(const KeyPlan& k, int64_t block) { return k.parts > 1 ? block : 0; }
__host__ __device__ inline int64_t far_slot(const KeyPlan& k, int kv_heads, int seq, int tile, int kvh, int part) {
  return (k.parts > 1 ? k.near_blocks : 0) + (((int64_t)seq * k.sink_tiles + tile) * kv_heads + kvh) * (k.far + 1) + part;
}

// Wavefronts of a block, and where they hold values.  bf16 heads of 128: eight, two a SIMD, so that one's arithmetic runs beside the other's products (one wavefront
// a SIMD with twice the rows issues them one after the other: 550 us where two take 440, window of 1024 in 2 x 4096 tokens, 32 heads of 128).  Four take
// the first 32 rows of a stage and four the second, for the same keys; the second ones' sums are added through LDS at the end.  They have
// no registers left for the values, which stay in LDS.  Smaller heads and fp32: four, each with all rows.
template <typename T, int DP>
struct DkvTile {
  static constexpr int WAVES = sizeof(T) == 2 && DP > 64 ? 8 : 4, BQ = sizeof(T) == 2 ? 64 : 32;
  static constexpr bool VALUES_IN_LDS = sizeof(T) == 2 && DP == 128;
};

// dk and dv of 128 keys, 32 a wavefront: scores with queries as rows and keys as columns, so that P and dS are operands of the sums over
// the queries where they are.
template <typename T, int DP>
__global__ __launch_bounds__((64 * DkvTile<T, DP>::WAVES), (kTwoWaves<T, DP> ? 2 : 1)) void k_attn_dkv(AttnArgs a, AttnGrads g, KeyPlan plan,
                                                                                              float* __restrict__ sums) {
  using R = RowTile<T, DP>;
  using C = DkvTile<T, DP>;
  constexpr int BQ = C::BQ, NW = C::WAVES, TILE = BQ * R::ROW, STAGE = 2 * TILE, VALUES = C::VALUES_IN_LDS ? kKeyRows * R::ROW : 0;
  __shared__ __attribute__((aligned(1024))) char smem[2 * STAGE + VALUES];
  __shared__ __attribute__((aligned(16))) float s_lse[2][BQ], s_delta[2][BQ];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kv_heads = a.heads / a.group;
  const bool far = blockIdx.x >= plan.near_blocks;                   // short ones, behind the others: they even out the end
  int seq, tile, kvh, part;
  int64_t slot;
  if (far) {
    int id = blockIdx.x - (int)plan.near_blocks;
    part = id % plan.far;
    id /= plan.far;
    kvh = id % kv_heads;
    id /= kv_heads;
    tile = id % plan.sink_tiles;
    seq = id / plan.sink_tiles;
    slot = far_slot(plan, kv_heads, seq, tile, kvh, part + 1);
  } else {
    const int id = xcd_contiguous_index(blockIdx.x, (int)plan.near_blocks);
    const int per_head = plan.tiles * plan.parts, at = id % per_head;
    kvh = id / per_head;
    part = at % plan.parts;
    if (!find_tile(a.ks, kKeyRows, at / plan.parts, &seq, &tile)) return;
    slot = near_slot(plan, id);
  }
  const int2 qp = a.qs.place(seq), kp = a.ks.place(seq);
  if (tile * kKeyRows >= kp.y) return;
  const bool near = plan.far > 0;                                    // what sinks add is not this block's, or all that is
  const int shift = kp.y - qp.y, own = wave & 3, sub = NW == 8 ? wave >> 2 : 0, k0 = tile * kKeyRows + own * 32, krow = k0 + (lane & 31);
  const QuerySpan span(a.mask, near && !far, qp.y, shift, tile * kKeyRows, min(tile * kKeyRows + kKeyRows, kp.y) - 1);
  const int nq = span.last > span.first ? (span.last - span.first + BQ - 1) / BQ : 0;
  const int cuts = far ? plan.far : plan.parts;
  const int begin = (int)((int64_t)nq * a.group * part / cuts), count = (int)((int64_t)nq * a.group * (part + 1) / cuts) - begin;
  // which pairs count: all that see each other; without sinks; sinks outside the window alone
  AttnMask mask = a.mask;
  if (near && !far) mask.sinks = 0;
  const AttnMask window_alone = {0, a.mask.window, 0};
  auto seen = [&](int p, int j) {
    const bool yes = mask.sees(p, j);
    return (bool)((int)yes & ((int)!far | ((int)(j < mask.sinks) & (int)!window_alone.sees(p, j))));
  };
  auto some = [&](int p0) { return mask.sees_some(p0, p0 + 31, k0, k0 + 31) && (!far || k0 < mask.sinks); };
  auto all = [&](int p0) { return !far && mask.sees_all(p0, p0 + 31, k0, k0 + 31); };

  RowCopies<T, DP, BQ, NW> cq(a.ldq, a.dim, wave), cd(g.lddo, a.dim, wave);
  float next_lse = 0.0f, next_delta = 0.0f;
  // stages are counted along the queries of a head, then along the heads: where the next copy, and the next scores, stand in that
  int to_head = kvh * a.group + (count > 0 ? begin / nq : 0), to_tile = count > 0 ? begin % nq : 0;
  int at_tile = to_tile;                             // of the stage that is worked on
  auto issue = [&](char* buf) {
    const int head = to_head, i0 = span.first + to_tile * BQ, valid = qp.y - i0;
    if (++to_tile == nq) {
      to_tile = 0;
      ++to_head;
    }
    cq.issue((const char*)((const T*)a.q + (int64_t)(qp.x + i0) * a.ldq + head * a.dim), valid, buf, wave);
    cd.issue((const char*)((const T*)g.dout + (int64_t)(qp.x + i0) * g.lddo + head * a.dim), valid, buf + TILE, wave);
    if (threadIdx.x < BQ) {
      const int i = threadIdx.x;
      const int64_t from = (int64_t)head * a.qs.rows + qp.x + i0 + i;
      next_lse = -INFINITY;                                         // rows behind the sequence are as tokens that see nothing
      next_delta = 0.0f;
      if (i < valid) {                                              // not looked at before keep(): that would wait for the copies too
        next_lse = g.lse[from];
        next_delta = g.delta[from];
      }
    }
  };
  auto keep = [&](int b) {
    if (threadIdx.x < BQ) {
      s_lse[b][threadIdx.x] = prob_base<T>(next_lse);
      s_delta[b][threadIdx.x] = next_delta;
    }
  };
  char* const vals = smem + 2 * STAGE;
  if constexpr (C::VALUES_IN_LDS) {
    const RowCopies<T, DP, kKeyRows, NW> cv(a.ldv, a.dim, wave);
    cv.issue((const char*)((const T*)a.v + ((int64_t)kp.x + tile * kKeyRows) * a.ldv + kvh * a.dim), kp.y - tile * kKeyRows, vals, wave, true);
  }
  if (count > 0) {
    issue(smem);
    keep(0);
  }
  const bool in = krow < kp.y;
  const int64_t row = (int64_t)kp.x + krow;
  Frag<T> k[R::KS], v[C::VALUES_IN_LDS ? 1 : R::KS];
#pragma unroll
  for (int ks = 0; ks < R::KS; ++ks) {
    const int c = 16 * ks + 8 * (lane >> 5);
    k[ks] = load_frag((const T*)a.k + row * a.ldk + kvh * a.dim + c, in && c < a.dim);
    if constexpr (!C::VALUES_IN_LDS) v[ks] = load_frag((const T*)a.v + row * a.ldv + kvh * a.dim + c, in && c < a.dim);
  }
  floatx16_t dk[R::ND], dv[R::ND];
#pragma unroll
  for (int i = 0; i < R::ND; ++i) dk[i] = dv[i] = zero16();
  const float c = prob_factor<T>(a.scale);
  tile_sync();
  for (int t = 0; t < count; ++t) {
    const int b = t & 1;
    if (t + 1 < count) issue(smem + (b ^ 1) * STAGE);
    const int stage_row = span.first + at_tile * BQ;
    if (++at_tile == nq) at_tile = 0;
#pragma unroll
    for (int n = 0; n < BQ / 32 * 4 / NW; ++n) {
      const int r0 = 32 * (sub + n), i0 = stage_row + r0, p0 = i0 + shift;
      const char *const qs = smem + b * STAGE + r0 * R::ROW, *const ds = qs + TILE;
      if (i0 < qp.y && some(p0)) {
        floatx16_t s = zero16(), dp = zero16();
#pragma unroll
        for (int ks = 0; ks < R::KS; ++ks) {
          mma(R::row_frag(qs, 0, ks), k[ks], s);
          if constexpr (C::VALUES_IN_LDS) mma(R::row_frag(ds, 0, ks), R::row_frag(vals, own * 32, ks), dp);
          else mma(R::row_frag(ds, 0, ks), v[ks], dp);
        }
        results_settle();
        if (!all(p0)) {
          const int first = p0 + row_here();
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] = seen(first + row_of(i), krow) ? s[i] : -INFINITY;
        }
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
          const float4 l4 = *(const float4*)&s_lse[b][r0 + result_row(i)], e4 = *(const float4*)&s_delta[b][r0 + result_row(i)];
          const float ls[4] = {l4.x, l4.y, l4.z, l4.w}, es[4] = {e4.x, e4.y, e4.z, e4.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i + j] = prob<T>(s[i + j], c, ls[j]);
            dp[i + j] = s[i + j] * (dp[i + j] - es[j]);
          }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const Frag<T> pf = frag_of<T>(s, h), df = frag_of<T>(dp, h);
#pragma unroll
          for (int i = 0; i < R::ND; ++i) {
            mma(R::col_frag(ds, 16 * h, i), pf, dv[i]);
            mma(R::col_frag(qs, 16 * h, i), df, dk[i]);
          }
        }
      }
    }
    if (t + 1 < count) keep(b ^ 1);
    tile_sync();
  }
  results_settle();
  if constexpr (NW == 8) {                           // the second four's sums, register by register
    static_assert(2 * STAGE >= 4 * R::ND * 16 * 64 * 4, "the sums lie where the stages were");
    float* const at = (float*)smem + own * (R::ND * 16 * 64) + lane;
    auto join = [&](floatx16_t (&x)[R::ND]) {
      if (sub == 1) {
#pragma unroll
        for (int i = 0; i < R::ND; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) at[(i * 16 + r) * 64] = x[i][r];
      }
      tile_sync();
      if (sub == 0) {
#pragma unroll
        for (int i = 0; i < R::ND; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) x[i][r] += at[(i * 16 + r) * 64];
      }
      tile_sync();
    };
    join(dk);
    join(dv);
    if (sub == 1) return;
  }
  const bool direct = plan.parts == 1 && !far && !(plan.far > 0 && tile < plan.sink_tiles);
  if (direct) {
    const int left = kp.y - k0;
    char* const place = smem + own * (2 * STAGE / kWaves);
    store_rows<T, DP>((T*)g.dk + ((int64_t)kp.x + k0) * g.lddk + kvh * a.dim, g.lddk, left, a.dim, dk, a.scale, place);
    store_rows<T, DP>((T*)g.dv + ((int64_t)kp.x + k0) * g.lddv + kvh * a.dim, g.lddv, left, a.dim, dv, 1.0f, place);
    return;
  }
  if (far && krow >= mask.sinks) return;             // nothing of theirs lies here
  if (!far && plan.parts == 1) slot = far_slot(plan, kv_heads, seq, tile, kvh, 0);
  constexpr int WIDTH = R::PITCH;
  float* to = sums + slot * (2 * kKeyRows * WIDTH) + (int64_t)(own * 32 + (lane & 31)) * WIDTH;
#pragma unroll
  for (int i = 0; i < R::ND; ++i) {
    store_col(to, dk[i], i, DP, a.scale);
    store_col(to + kKeyRows * WIDTH, dv[i], i, DP, 1.0f);
  }
}

// The sums of a tile's parts added in their order, those of the sinks' rows with their far parts.  Blocks: the tiles, or (where tiles are not
// cut) those with sinks; sixteen for the rows of one.
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_dkv_join(AttnArgs a, AttnGrads g, KeyPlan plan, const float* __restrict__ sums) {
  const int kv_heads = a.heads / a.group, id = blockIdx.x, kvh = id % kv_heads;
  int seq, tile;
  if (plan.parts > 1) {
    if (!find_tile(a.ks, kKeyRows, id / kv_heads, &seq, &tile)) return;
  } else {
    seq = id / kv_heads / plan.sink_tiles;
    tile = id / kv_heads - seq * plan.sink_tiles;
  }
  const int2 kp = a.ks.place(seq);
  const bool sinks = plan.far > 0 && tile < plan.sink_tiles;
  const int near = plan.parts;
  // near parts of the tile are neighbours among those of the head, or alone before the far ones
  const int64_t base = near > 1 ? ((int64_t)kvh * plan.tiles + id / kv_heads) * near : far_slot(plan, kv_heads, seq, tile, kvh, 0);
  const int64_t far = sinks ? far_slot(plan, kv_heads, seq, tile, kvh, 1) : 0;
  constexpr int PER_ROW = DP / 4, ROWS = 256 / PER_ROW;              // four features a lane
  for (int r = blockIdx.y * ROWS + threadIdx.x / PER_ROW; r < 2 * kKeyRows; r += gridDim.y * ROWS) {
    const int d = threadIdx.x % PER_ROW * 4, krow = tile * kKeyRows + r % kKeyRows;
    if (krow >= kp.y || d >= a.dim) continue;
    const int parts = near + (sinks && krow < a.mask.sinks ? plan.far : 0);
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll 4
    for (int x = 0; x < parts; ++x) {
      const int64_t slot = x < near ? base + x : far + x - near;
      const float4 v = *(const float4*)(sums + (slot * 2 * kKeyRows + r) * DP + d);
      sum.x += v.x;
      sum.y += v.y;
      sum.z += v.z;
      sum.w += v.w;
    }
    T* to = r < kKeyRows ? (T*)g.dk + ((int64_t)kp.x + krow) * g.lddk : (T*)g.dv + ((int64_t)kp.x + krow) * g.lddv;
    store4(to + kvh * a.dim + d, sum.x, sum.y, sum.z, sum.w);
  }
}

// far parts where a window's tiles have less to do than a tile with sinks, and few enough tiles that the chip does not fill by them; parts
// where tiles do not fill it.  The lengths are data of the device: both go by their mean.  Backward alone, us, chosen rule last:
//   parts, two blocks a CU      1 x 2048 tokens, 32 / 8 heads of 128: whole tiles 362, 256 blocks 255, 1024 blocks 249, 512 blocks 221;  1 x 1024: 186,
//                               108, 141, 110;  1 x 4096, 16 / 4 of 64: 597, 374, 262, 264;  fp32, 4 x 1000, 6 / 2 of 80: 865, 363, 335, 303
//   four steps a part at least  1 x 300, 4 / 2 of 64: whole 38.9, two steps 28.0, eight 33.3, four 30.8;  no difference in the sizes above
//   whole from 256 blocks on    8 x 384, 12 of 64 (288 blocks): cut 59, whole 43;  1 x 4096, 32 / 8 of 128 (256 blocks): cut 644, whole 831 (tiles
//                               of long causal sequences are uneven, which the rule does not look at)
//   far parts, one a CU         2 x 4096, 32 / 8 of 128, W 1024: none 1038, 128 of them 700, 512 662, 256 671;  1 x 16384, W 512: 3457, 974, 908, 900;
//                               16 x 2048, 12 of 64, W 256: 453, 387, 351, 337;  1 x 8192, 8 of 64, W 64, 300 sinks: 377, 125, 88, 98
//   eight steps a far part      the last one: four 98, sixteen 111, eight 98;  fp32, 2 x 3000, 6 / 2 of 80, W 500: 515, 575, 505
//   none from 256 tiles with sinks on  24 x 2048, 12 of 64, W 256 (288 of them): with far parts 535, without 648
static KeyPlan key_plan(const Packed& qs, const Packed& ks, int64_t kv_heads, int64_t group, const AttnMask& m, int dtype) {
  KeyPlan k = {};
  const int64_t tiles = ks.most_tiles(kKeyRows), stage = dtype == EFQAT_BF16 ? 64 : 32, each = ceil_div(qs.rows, qs.n);
  int64_t span = m.window && m.window + kKeyRows < each ? m.window + kKeyRows : each;      // queries of a tile
  const int64_t steps = ceil_div(span, stage) * group, blocks = tiles * kv_heads;
  int64_t parts = ceil_div(512, blocks);
  if (blocks >= 256) parts = 1;
  if (parts > ceil_div(steps, 4)) parts = ceil_div(steps, 4);
  k.tiles = (int)tiles;
  k.parts = (int)(parts < 1 ? 1 : parts);
  if (m.window && m.sinks > 0 && each > 2 * span) {
    const int64_t sink_tiles = ceil_div(m.sinks < ks.rows ? m.sinks : ks.rows, kKeyRows), sink_blocks = sink_tiles * qs.n * kv_heads;
    if (sink_blocks < 256) {
      const int64_t most = ceil_div(ceil_div(each - span, stage) * group, 8), want = ceil_div(256, sink_blocks);
      k.sink_tiles = (int)sink_tiles;
      k.far = (int)(most < want ? most : want);
      k.far_blocks = sink_blocks * k.far;
    }
  }
  k.near_blocks = blocks * k.parts;
  k.slots = (k.parts > 1 ? k.near_blocks : 0) + (k.far ? k.far_blocks / k.far * (k.far + 1) : 0);
  return k;
}

}  // namespace efqat

using namespace efqat;

static size_t bwd_ws_bytes(const KeyPlan& k, int64_t Tq, int64_t heads, int64_t dim) {
  return (size_t)round_up(Tq * heads * 4, 256) + (size_t)k.slots * 2 * kKeyRows * (dim <= 64 ? 64 : 128) * 4;
}

extern "C" size_t efqat_attention_bwd_workspace_bytes(int64_t Tq, int64_t Tk, int64_t n_seq, int packed, int64_t heads, int64_t kv_heads, int64_t dim,
                                                      int dtype, int causal, int64_t window, int64_t sinks) {
  AttnArgs a;
  static const int32_t some[1] = {0};
  void* const p = (void*)16;                         // any pointer and stride that would do
  if (attn_args(&a, p, heads * dim, p, kv_heads * dim, p, kv_heads * dim, dtype, Tq, Tk, n_seq, packed ? some : nullptr, packed ? some : nullptr, heads,
                kv_heads, dim, 1.0f, causal, window, sinks))
    return 256;
  return bwd_ws_bytes(key_plan(a.qs, a.ks, kv_heads, a.group, a.mask, dtype), Tq, heads, dim);
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
  const KeyPlan plan = key_plan(a.qs, a.ks, kv_heads, a.group, a.mask, dtype);
  if (ws_bytes < bwd_ws_bytes(plan, Tq, heads, dim)) return EFQAT_ERR_WORKSPACE;
  const HeadPlan h = head_plan(a, kv_heads);
  const int64_t key_waves = (plan.near_blocks + plan.far_blocks) * (dtype == EFQAT_BF16 && dim > 64 ? DkvTile<bf16_t, 128>::WAVES : DkvTile<bf16_t, 64>::WAVES);
  static_assert(DkvTile<bf16_t, 96>::WAVES == DkvTile<bf16_t, 128>::WAVES && DkvTile<float, 128>::WAVES == DkvTile<bf16_t, 64>::WAVES, "as counted above");
  if (h.blocks > kAttnMostBlocks || key_waves > kAttnMostBlocks * 4) return EFQAT_ERR_BAD_SHAPE;
  EFQAT_TRY(attn_apart({dq, dk, dv}, {q, k, v, dout, o}));
  EFQAT_TRY(attn_apart({dq}, {dk, dv}));
  EFQAT_TRY(attn_apart({dk}, {dv}));
  const AttnGrads g = {dout, o, lddo, ldo, lse, (float*)ws, dq, dk, dv, lddq, lddk, lddv};
  float* sums = (float*)((char*)ws + round_up(Tq * heads * 4, 256));
  const unsigned joins = (unsigned)(plan.parts > 1 ? plan.tiles * kv_heads : plan.far ? plan.far_blocks / plan.far : 0);
  hipStream_t st = (hipStream_t)stream;
#define EFQAT_BWD(E, DP)                                                                                                           \
  do {                                                                                                                             \
    EFQAT_TRY(launch(k_attn_dq<E, DP>, dim3((unsigned)h.blocks), dim3(256), 0, st, a, g, h.tiles, h.hb));                          \
    EFQAT_TRY(launch(k_attn_dkv<E, DP>, dim3((unsigned)(plan.near_blocks + plan.far_blocks)), dim3(64 * DkvTile<E, DP>::WAVES), 0, st, a, g, plan, sums)); \
    if (joins) EFQAT_TRY(launch(k_attn_dkv_join<E, RowTile<E, DP>::PITCH>, dim3(joins, 16), dim3(256), 0, st, a, g, plan, (const float*)sums));        \
    return EFQAT_OK;                                                                                                               \
  } while (0)
  if (dtype == EFQAT_F32) { if (dim <= 64) EFQAT_BWD(float, 64); if (dim <= 96) EFQAT_BWD(float, 96); EFQAT_BWD(float, 128); }
  if (dim <= 64) EFQAT_BWD(bf16_t, 64);
  if (dim <= 96) EFQAT_BWD(bf16_t, 96);
  EFQAT_BWD(bf16_t, 128);
#undef EFQAT_BWD
}
