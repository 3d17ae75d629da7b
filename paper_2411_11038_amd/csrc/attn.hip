// Attention with a sliding window and first tokens that stay visible, forward, and its form for one new token a sequence.
//
//   s_ij = scale q_i . k_j over the keys that token i sees,  m_i = max_j s_ij,  l_i = sum_j exp(s_ij - m_i),
//   o_i = sum_j exp(s_ij - m_i) v_j / l_i,  lse_i = m_i + log l_i
//
// One pass over the keys: with a new largest score m', l and o are multiplied by exp(m - m').  Scores are formed transposed, keys as
// rows and queries as columns of a result: a lane then holds 16 scores of one query, its maximum and sum need one exchange between the
// halves of a wavefront, and the probabilities are the second product's operand where they are.  With bf16 they are rounded to it there, to
// nearest: the fp32 product would take sixteen times as long, and half a step of each of many terms is less in o than o's own (o is off by 1.8e-3 to
// 2.1e-3 in the 2-norm, where rounding the exact result is 1.66e-3).  l sums them before they are rounded.
//
// Bound by the matrix cores and the power limit: 32768 tokens, 32 query and 8 key heads of 128, causal, 7.8 ms (1.12 PFLOP/s, where
// a library product of 8192^3 reaches 1.41 on the same card; another card: 8.1); with zero operands 5.93 ms; a window of 1024 in 2 x 4096 tokens 169 us;
// 32 x 384 tokens, 12 heads of 64, 37 us, where a block has six tiles.  Blocks come from the queries alone: 16 tokens over 32768 keys are 8 blocks, 600 us.
// Single tokens are bound by HBM: 64 sequences of 500 to 8192 keys, 8 key heads of 128, 222 to 230 us (5.0 TB/s), one of 16384 keys 17 us and 4 for
// the join; fp32, where heads beyond 64 have one stage of LDS: the same sequence 39 us in all, 32 of 512 to 8192 keys 311 us (3.9 TB/s).
#include "attn_tile.hpp"

namespace efqat {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.69314718055994531f, kLn2Rest = -1.9046542999e-9f;      // ln 2 = kLn2 + kLn2Rest

// exp2(s c - m c) in one operation beside the exponential lacks what rounding took from m c, a factor that all of a row share.  Beyond this it
// would leave the range of fp32: m is taken from the scores first.
constexpr float kFarBase = 65536.0f;
// what sums with reference m are worth beside the largest reference
__device__ __forceinline__ float decay(float m, float top, float c) { return top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - top) * c); }

// log of l exp2(m c), the sum that l stands for: m c as it was rounded where l was summed.  Where m c leaves fp32 (scores beyond 2.36e38, log2 e short of
// its end) both parts of ln 2 would meet as infinities of opposite signs: m scale is formed instead.  A row whose l is not a number has no lse either.
__device__ __forceinline__ float log_sum(float m, float c, float scale, float l) {
  const float base = m == -INFINITY ? 0.0f : m * c;            // a factor so small that no score passes it: m has not moved
  if (l == 0.0f) return -INFINITY;
  const float rest = kLn2 * __builtin_amdgcn_logf(l);
  if (fabsf(base) == INFINITY) return fmaf(m, scale, rest);
  return fmaf(base, kLn2, fmaf(base, kLn2Rest, rest));
}

template <int NT>
__device__ __forceinline__ float max_of(const floatx16_t (&s)[NT]) {
  float top = -INFINITY;
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
  return top;
}
// scores of a wavefront's 32 queries (columns) against BN keys; what is not seen is -inf
template <int NT>
__device__ __forceinline__ void mask_scores(floatx16_t (&s)[NT], const AttnMask& m, int p, int j0, int end) {
  j0 += row_here();
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = j0 + 32 * n + row_of(i);
      s[n][i] = ((j < end) & m.sees(p, j)) ? s[n][i] : -INFINITY;
    }
}

// A block takes 128 rows of scores: `hb` of the heads that share keys, 128 / hb queries of each.  (256 rows halve what L2 delivers, but
// their eight wavefronts wait for each other: no faster at 32768 tokens, a third slower at 384.)
//
// A lane's maximum is not followed exactly: l and o refer to the score m, which moves only where a score passes it by 8 / log2 e, so that
// probabilities stay below 2^8 and the accumulators are hardly ever multiplied.
template <typename T, int DP>
__global__ __launch_bounds__(256, (kTwoWaves<T, DP> ? 2 : 1)) void k_attn_fwd(AttnArgs a, T* __restrict__ o, int64_t ldo,
                                                                                         float* __restrict__ lse, int tiles, int hb) {
  using R = RowTile<T, DP>;
  constexpr int BN = kKeyStage<T>, NT = BN / 32, TILE = BN * R::ROW;
  __shared__ __attribute__((aligned(1024))) char smem[4 * TILE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  HeadTile w;
  if (!w.find(a, hb, tiles, wave)) return;
  const int p = w.row + (lane & 31) + w.shift;
  const KeyTiles kt(a.mask, w.keys.y, w.block_row + w.shift, w.block_row + w.block_rows - 1 + w.shift, BN);
  KeyCopies<T, DP, BN> copies(a, w.keys, w.kvh, wave);

  Frag<T> q[R::KS];
  {
    const T* row = (const T*)a.q + w.token(lane) * a.ldq + w.head * a.dim;
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks) {
      const int d = 16 * ks + 8 * (lane >> 5);
      q[ks] = load_frag(row + d, w.in(lane) && d < a.dim);
    }
  }
  floatx16_t acc[R::ND];
#pragma unroll
  for (int i = 0; i < R::ND; ++i) acc[i] = zero16();
  float m = -INFINITY, l = 0.0f;
  const float c = a.scale * kLog2e, slack = 8.0f / c;

  // Keys are a tile ahead of values: while tile t's scores become probabilities, the scores of tile t + 1 are formed.  Two places in LDS for
  // keys, two for values; what was copied during a step is there at its end.
  char* const vals = smem + 2 * TILE;
  float top = -INFINITY;
  // scores of the tile whose keys lie at `keys`, and beside each product a share of tile t's probabilities, as operands of the next product
  auto scores = [&](const char* keys, floatx16_t (&u)[NT], floatx16_t (&s)[NT], Frag<T> (&pf)[2 * NT], float base, auto both) {
    constexpr int GROUPS = R::KS * NT;
    Frag<T> kf[2][NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      u[n] = zero16();
      kf[0][n] = R::row_frag(keys, 32 * n, 0);
    }
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks)
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if (ks + 1 < R::KS) kf[(ks + 1) & 1][n] = R::row_frag(keys, 32 * n, ks + 1);
        mma(kf[ks & 1][n], q[ks], u[n]);
        if constexpr (decltype(both)::value) {
#pragma unroll
          for (int e = (ks * NT + n) * 16 * NT / GROUPS; e < (ks * NT + n + 1) * 16 * NT / GROUPS; ++e) {
            s[e >> 4][e & 15] = __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], c, -base));
            if ((e & 7) == 7) {
              l += sum8(s[e >> 4], (e >> 3) & 1);
              pf[e >> 3] = frag_of<T>(s[e >> 4], (e >> 3) & 1);
              hold(pf[e >> 3]);
            }
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    top = max_of(u);
    hold(top);                                       // all results are read here, before a branch
  };
  auto hide = [&](int t, floatx16_t (&u)[NT]) {
    const int j0 = kt.tile(t) * BN, p0 = w.row + w.shift;
    if (j0 + BN > w.keys.y || !a.mask.sees_all(p0, p0 + 31, j0, j0 + BN - 1)) {
      mask_scores(u, a.mask, p, j0, w.keys.y);
      top = max_of(u);
    }
  };
  auto step = [&](int t, floatx16_t (&s)[NT], floatx16_t (&u)[NT]) {
    if (t + 2 < kt.count) copies.issue_keys(kt.tile(t + 2), smem + (t & 1) * TILE, wave);
    if (t + 1 < kt.count) copies.issue_values(kt.tile(t + 1), vals + ((t + 1) & 1) * TILE, wave);
    top = half_max(top);
    if (__any(top > m + slack)) {
      results_settle();
      const float next = fmaxf(m, top);
      const float shrink = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - next) * c);
      m = next;
      l *= shrink;
#pragma unroll
      for (int i = 0; i < R::ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] *= shrink;
    }
    float base = m == -INFINITY ? 0.0f : m * c;                    // nothing seen so far: exp2(-inf) is 0 for all of it
    if (__any(fabsf(base) > kFarBase)) {
      const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[n][i] -= ref;
      base = 0.0f;
    }
    Frag<T> pf[2 * NT];
    scores(smem + ((t + 1) & 1) * TILE, u, s, pf, base, std::true_type{});      // behind the last tile: of what lies there, not used
    if (t + 1 < kt.count) hide(t + 1, u);
    // values are read a step ahead of the products that take them
    const char* at = vals + (t & 1) * TILE;
    Frag<T> v[2][R::ND];
#pragma unroll
    for (int i = 0; i < R::ND; ++i) v[0][i] = R::col_frag(at, 0, i);
#pragma unroll
    for (int x = 0; x < 2 * NT; ++x) {
      if (x + 1 < 2 * NT) {
#pragma unroll
        for (int i = 0; i < R::ND; ++i) v[(x + 1) & 1][i] = R::col_frag(at, 16 * (x + 1), i);
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < R::ND; ++i) mma(v[x & 1][i], pf[x], acc[i]);
    }
    tile_sync();
  };
  if (kt.count > 0) {
    floatx16_t s[NT], u[NT];
    Frag<T> none[2 * NT];
    copies.issue_keys(kt.tile(0), smem, wave);
    tile_sync();
    if (kt.count > 1) copies.issue_keys(kt.tile(1), smem + TILE, wave);
    copies.issue_values(kt.tile(0), vals, wave);
    scores(smem, s, u, none, 0.0f, std::false_type{});
    hide(0, s);
    tile_sync();
    for (int t = 0;; t += 2) {
      step(t, s, u);
      if (t + 1 >= kt.count) break;
      step(t + 1, u, s);
      if (t + 2 >= kt.count) break;
    }
  }
  results_settle();
  l = half_sum(l);
  const float f = l == 0.0f ? 0.0f : 1.0f / l;                     // a token that sees nothing: zeros
  store_rows<T, DP>(o + w.token(0) * ldo + w.head * a.dim, ldo, w.rows_left(), a.dim, acc, f, smem + wave * (sizeof(smem) / kWaves));
  if (lse && lane < 32 && w.in(lane)) lse[(int64_t)w.head * a.qs.rows + w.token(lane)] = log_sum(m, c, a.scale, l);
}

// ---- one new token a sequence
// A block takes one sequence, one key head with up to 32 of its query heads (the columns of a result) and a share of the keys;
// its wavefronts take 32 keys at a time by themselves, each with its own part of LDS, and are joined at the end.  Shares of more
// than one block are joined by k_attn_join.
struct DecodeArgs {
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv, seq_k, seq_v;
  const int32_t* lengths;
  int capacity, heads, group, dim, window, sinks, splits;
  float scale;
};

template <typename T, int DP>
struct DecodeTile {
  using R = RowTile<T, DP>;
  static constexpr int BN = 32, STAGE = 2 * BN * R::ROW, STAGES = sizeof(T) == 2 || DP <= 64 ? 2 : 1;
  static constexpr int LDS = 4 * STAGE * STAGES;
};

template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_decode(DecodeArgs a, T* __restrict__ o, int64_t ldo, float* __restrict__ part) {
  using C = DecodeTile<T, DP>;
  using R = RowTile<T, DP>;
  constexpr int BN = C::BN, COPIES = 2 * BN / R::RPI;                    // of a stage, in flight behind the one that is waited for
  __shared__ __attribute__((aligned(1024))) char smem[C::LDS];
  __shared__ float s_m[4][32], s_l[4][32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int split = blockIdx.x, seq = blockIdx.z, row_tiles = (a.group + 31) / 32;
  const int kvh = blockIdx.y / row_tiles, g0 = (blockIdx.y - kvh * row_tiles) * 32, g = g0 + (lane & 31);
  int keys = a.lengths[seq];
  keys = keys < 0 ? 0 : keys > a.capacity ? a.capacity : keys;
  const AttnMask mask = {1, a.window, a.sinks};
  const int p = keys - 1;
  const KeyTiles kt(mask, keys, p, p, BN);
  const int first = (int)((int64_t)kt.count * split / a.splits), last = (int)((int64_t)kt.count * (split + 1) / a.splits);

  const char* kbase = (const char*)((const T*)a.k + seq * a.seq_k + kvh * a.dim);
  const char* vbase = (const char*)((const T*)a.v + seq * a.seq_v + kvh * a.dim);
  const int64_t ldk = a.ldk * (int)sizeof(T), ldv = a.ldv * (int)sizeof(T);
  const int pieces = a.dim * (int)sizeof(T) / 16;
  char* own = smem + wave * C::STAGE * C::STAGES;
  auto issue_keys = [&](int t, char* buf) {
    const int j0 = kt.tile(t) * BN, valid = keys - j0;
#pragma unroll
    for (int s = 0; s < BN / R::RPI; ++s) R::copy(kbase + j0 * ldk, ldk, valid, pieces, buf, s);
  };
  auto issue_values = [&](int t, char* buf) {
    const int j0 = kt.tile(t) * BN, valid = keys - j0;
#pragma unroll
    for (int s = 0; s < BN / R::RPI; ++s) R::copy(vbase + j0 * ldv, ldv, valid, pieces, buf + BN * R::ROW, s);
  };
  Frag<T> q[R::KS];
  {
    const T* row = (const T*)a.q + seq * a.ldq + (int64_t)(kvh * a.group + g) * a.dim;
#pragma unroll
    for (int ks = 0; ks < R::KS; ++ks) {
      const int d = 16 * ks + 8 * (lane >> 5);
      q[ks] = load_frag(row + d, g < a.group && d < a.dim);
    }
  }
  floatx16_t acc[R::ND];
#pragma unroll
  for (int i = 0; i < R::ND; ++i) acc[i] = zero16();
  float m = -INFINITY, l = 0.0f;
  const float c = a.scale * kLog2e;
  // Two stages: the next tile is copied while one is worked on.  One (where two do not fit): the next keys are, from when the scores are formed,
  // and the next values behind the products.
  constexpr int HALF = COPIES / 2;
  auto arrived = [&](bool behind, auto left) {       // all copies but the last `left`, if so many were issued behind what is waited for
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
    if (behind) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(left)::value) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#endif
  };
  auto was_read = [&]() {                            // a tile in LDS: the next copies may overwrite it
#if defined(__HIP_DEVICE_COMPILE__)
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
#endif
  };
  int n = 0;
  if (first + wave < last) {
    issue_keys(first + wave, own);
    issue_values(first + wave, own);
  }
  for (int t = first + wave; t < last; t += 4, ++n) {
    char* buf = own + (C::STAGES == 2 ? (n & 1) * C::STAGE : 0);
    const bool more = t + 4 < last;
    if constexpr (C::STAGES == 2) {
      if (more) {
        issue_keys(t + 4, own + ((n + 1) & 1) * C::STAGE);
        issue_values(t + 4, own + ((n + 1) & 1) * C::STAGE);
      }
      arrived(more, std::integral_constant<int, COPIES>{});
    } else {
      arrived(true, std::integral_constant<int, HALF>{});            // the values of this tile may be on their way
    }
    const int j0 = kt.tile(t) * BN;
    auto tile = [&](auto masked) {
      floatx16_t s[1] = {zero16()};
#pragma unroll
      for (int ks = 0; ks < R::KS; ++ks) mma(R::row_frag(buf, 0, ks), q[ks], s[0]);
      if constexpr (decltype(masked)::value) mask_scores(s, mask, p, j0, keys);
      float top = m;
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[0][i]);
      if constexpr (C::STAGES == 1) {
        hold(top);                                   // all results are read here, before the branch
        was_read();
        if (more) issue_keys(t + 4, buf);
      }
      top = half_max(top);
      const float ref = top == -INFINITY ? 0.0f : top, shrink = __builtin_amdgcn_exp2f((m - ref) * c);
      m = top;
#pragma unroll
      for (int i = 0; i < R::ND; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] *= shrink;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[0][i] = __builtin_amdgcn_exp2f((s[0][i] - ref) * c);
      l = fmaf(l, shrink, sum16(s[0]));
      if constexpr (C::STAGES == 1) arrived(more, std::integral_constant<int, HALF>{});
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const Frag<T> pf = frag_of<T>(s[0], h);
#pragma unroll
        for (int i = 0; i < R::ND; ++i) mma(R::col_frag(buf + BN * R::ROW, 16 * h, i), pf, acc[i]);
      }
    };
    if (mask.sees_all(p, p, j0, j0 + BN - 1)) tile(std::false_type{});
    else tile(std::true_type{});
    was_read();
    if (C::STAGES == 1 && more) issue_values(t + 4, buf);
  }
  results_settle();
  l = half_sum(l);
  if (lane < 32) {
    s_m[wave][lane] = m;
    s_l[wave][lane] = l;
  }
  tile_sync();
  // the wavefronts' outputs on a common base, [wave][column][WIDTH] in the tiles' place (columns one bank apart)
  constexpr int WIDTH = R::PITCH, PITCH = WIDTH + 4;
  static_assert(4 * 32 * PITCH * 4 <= C::LDS, "the joined columns lie where the tiles were");
  float top = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) top = fmaxf(top, s_m[w][lane & 31]);
  float* mine = (float*)smem + (wave * 32 + (lane & 31)) * PITCH;
  const float f = decay(m, top, c);
#pragma unroll
  for (int i = 0; i < R::ND; ++i) store_col(mine, acc[i], i, WIDTH, f);
  tile_sync();
  const int cols = min(32, a.group - g0);
  for (int e = threadIdx.x; e < cols * (WIDTH / 4); e += 256) {
    const int col = e / (WIDTH / 4), d = (e - col * (WIDTH / 4)) * 4;
    if (d >= DP) continue;
    float tm = -INFINITY, tl = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) tm = fmaxf(tm, s_m[w][col]);
    float4 sum = make_float4(0, 0, 0, 0);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      tl += s_l[w][col] * decay(s_m[w][col], tm, c);
      const float4 v = *(const float4*)((const float*)smem + (w * 32 + col) * PITCH + d);
      sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    const int head = kvh * a.group + g0 + col;
    if (a.splits == 1) {
      const float r = tl == 0.0f ? 0.0f : 1.0f / tl;
      if (d < a.dim) store4(o + seq * ldo + (int64_t)head * a.dim + d, sum.x * r, sum.y * r, sum.z * r, sum.w * r);
    } else {
      float* to = part + (((int64_t)seq * a.heads + head) * a.splits + split) * (WIDTH + 4);
      *(float4*)(to + d) = sum;
      if (d == 0) *(float4*)(to + WIDTH) = make_float4(tm, tl, 0, 0);
    }
  }
}

// The shares of a head's keys put together: a block for each sequence and head, its wavefronts every fourth share.  All that a share leaves is
// read at once; their weights are made by a lane each.
constexpr int kMostShares = 64;
template <typename T, int DP>
__global__ __launch_bounds__(256) void k_attn_join(const float* __restrict__ part, int splits, int heads, int dim, float c, T* __restrict__ o,
                                                   int64_t ldo) {
  constexpr int PER = DP / 64;
  __shared__ float s_sum[3][DP];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, head = blockIdx.x, seq = blockIdx.y;
  const float* from = part + ((int64_t)seq * heads + head) * splits * (DP + 4);
  const float m = lane < splits ? from[lane * (DP + 4) + DP] : -INFINITY, l = lane < splits ? from[lane * (DP + 4) + DP + 1] : 0.0f;
  float v[kMostShares / 4][PER];
#pragma unroll
  for (int x = 0; x < kMostShares / 4; ++x) {
    const int s = wave + 4 * x;
#pragma unroll
    for (int i = 0; i < PER; ++i) v[x][i] = s < splits ? from[s * (DP + 4) + lane * PER + i] : 0.0f;
  }
  const float f = decay(m, wave_max(m), c), total = wave_total(l * f);
  float sum[PER] = {};
#pragma unroll
  for (int x = 0; x < kMostShares / 4; ++x) {
    const float w = __shfl(f, wave + 4 * x, 64);
#pragma unroll
    for (int i = 0; i < PER; ++i) sum[i] = fmaf(v[x][i], w, sum[i]);
  }
  if (wave > 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) s_sum[wave - 1][lane * PER + i] = sum[i];
  }
  __syncthreads();
  if (wave == 0) {
    const float r = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int d = lane * PER + i;
      sum[i] = ((sum[i] + s_sum[0][d]) + (s_sum[1][d] + s_sum[2][d])) * r;
      if (d < dim) o[seq * ldo + (int64_t)head * dim + d] = from_f32<T>(sum[i]);
    }
  }
}

static int attn_dp(int64_t dim) { return dim <= 64 ? 64 : 128; }

// Shares of a sequence's keys: as many blocks as the chip has CUs, one for every sixteen tiles of 32 keys at most (rounded up: 17 tiles are
// two shares of eight and nine, 512 are 32 of four tiles a wavefront), and eight a CU where shares stay long, 64 tiles at least (sequences differ in length: 64 of 500 to 8192 keys, 8 heads of 128, 248 us in one share, 224 in four; 24 of 1028 keys, 12
// heads of 64, 20 us in one, 24 in two).
static int decode_splits(int64_t n_seq, int64_t capacity, int64_t heads, int64_t kv_heads, int64_t window, int64_t sinks) {
  const int64_t most = window > 0 && window < capacity && sinks < capacity && window + sinks + 64 < capacity ? window + sinks + 64 : capacity;
  const int64_t tiles = ceil_div(most, 32), blocks = n_seq * kv_heads * ceil_div(heads / kv_heads, 32);
  auto at_most = [](int64_t a, int64_t b) { return a < b ? a : b; };
  const int64_t fill = at_most(ceil_div(256, blocks), ceil_div(tiles, 16)), even = at_most(ceil_div(2048, blocks), tiles / 64);
  const int64_t s = at_most(fill > even ? fill : even, kMostShares);
  return (int)(s < 1 ? 1 : s);
}

}  // namespace efqat

using namespace efqat;

extern "C" int efqat_attention_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int dtype, int64_t Tq,
                                   int64_t Tk, int64_t n_seq, const int32_t* q_start, const int32_t* k_start, int64_t heads,
                                   int64_t kv_heads, int64_t dim, float scale, int causal, int64_t window, int64_t sinks, void* o,
                                   int64_t ldo, float* lse, void* stream) {
  AttnArgs a;
  EFQAT_TRY(attn_args(&a, q, ldq, k, ldk, v, ldv, dtype, Tq, Tk, n_seq, q_start, k_start, heads, kv_heads, dim, scale, causal, window, sinks));
  EFQAT_TRY(attn_rows(o, ldo, heads * dim, dtype));
  if (!aligned4(lse)) return EFQAT_ERR_ALIGNMENT;
  const HeadPlan h = head_plan(a, kv_heads);
  if (h.blocks > kAttnMostBlocks) return EFQAT_ERR_BAD_SHAPE;
  EFQAT_TRY(attn_apart({o}, {q, k, v}));
  hipStream_t st = (hipStream_t)stream;
#define EFQAT_FWD(E, DP) return launch(k_attn_fwd<E, DP>, dim3((unsigned)h.blocks), dim3(256), 0, st, a, (E*)o, ldo, lse, h.tiles, h.hb)
  if (dtype == EFQAT_F32) { if (dim <= 64) EFQAT_FWD(float, 64); if (dim <= 96) EFQAT_FWD(float, 96); EFQAT_FWD(float, 128); }
  if (dim <= 64) EFQAT_FWD(bf16_t, 64);
  if (dim <= 96) EFQAT_FWD(bf16_t, 96);
  EFQAT_FWD(bf16_t, 128);
#undef EFQAT_FWD
}

extern "C" size_t efqat_attention_decode_workspace_bytes(int64_t n_seq, int64_t capacity, int64_t heads, int64_t kv_heads, int64_t dim,
                                                         int64_t window, int64_t sinks) {
  if (n_seq <= 0 || capacity <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || dim <= 0 || dim > 128 || window < 0 || sinks < 0 ||
      n_seq > 65535 || capacity > kAttnMostRows || heads > 65535)
    return 256;
  const int splits = decode_splits(n_seq, capacity, heads, kv_heads, window, sinks);
  if (splits == 1) return 256;
  return (size_t)round_up(n_seq * heads * splits * (attn_dp(dim) + 4) * 4, 256);
}

extern "C" int efqat_attention_decode(const void* q, int64_t ldq, const void* k_cache, int64_t ldk, int64_t seq_k, const void* v_cache,
                                      int64_t ldv, int64_t seq_v, int dtype, int64_t n_seq, int64_t capacity, const int32_t* lengths,
                                      int64_t heads, int64_t kv_heads, int64_t dim, float scale, int64_t window, int64_t sinks, void* o,
                                      int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  AttnArgs a;
  EFQAT_TRY(attn_args(&a, q, ldq, k_cache, ldk, v_cache, ldv, dtype, n_seq, capacity, 1, nullptr, nullptr, heads, kv_heads, dim, scale, 1, window, sinks));
  EFQAT_TRY(attn_rows(o, ldo, heads * dim, dtype));
  if (n_seq > 65535 || (n_seq > 1 && (seq_k < 0 || seq_v < 0))) return EFQAT_ERR_BAD_SHAPE;
  if (!lengths || !ws) return EFQAT_ERR_NULL_PTR;
  if (!aligned4(lengths) || (uintptr_t)ws % 256) return EFQAT_ERR_ALIGNMENT;
  const int per16 = dtype == EFQAT_F32 ? 4 : 8;
  if (n_seq > 1 && (seq_k % per16 || seq_v % per16)) return EFQAT_ERR_ALIGNMENT;
  if (ws_bytes < efqat_attention_decode_workspace_bytes(n_seq, capacity, heads, kv_heads, dim, window, sinks)) return EFQAT_ERR_WORKSPACE;
  EFQAT_TRY(attn_apart({o}, {q, k_cache, v_cache}));
  const int splits = decode_splits(n_seq, capacity, heads, kv_heads, window, sinks);
  const DecodeArgs d = {q, k_cache, v_cache, ldq, ldk, ldv, n_seq > 1 ? seq_k : 0, n_seq > 1 ? seq_v : 0, lengths, (int)capacity, (int)heads,
                        a.group, (int)dim, a.mask.window, a.mask.sinks, splits, scale};
  const int64_t ny = kv_heads * ceil_div(a.group, 32);
  const dim3 grid((unsigned)splits, (unsigned)ny, (unsigned)n_seq);
  hipStream_t st = (hipStream_t)stream;
  float* part = (float*)ws;
#define EFQAT_DEC(E, DP)                                                                                                           \
  do {                                                                                                                             \
    EFQAT_TRY(launch(k_attn_decode<E, DP>, grid, dim3(256), 0, st, d, (E*)o, ldo, part));                                          \
    if (splits > 1)                                                                                                                \
      EFQAT_TRY(launch(k_attn_join<E, RowTile<E, DP>::PITCH>, dim3((unsigned)heads, (unsigned)n_seq), dim3(256), 0, st, part, splits, (int)heads,      \
                       (int)dim, scale * kLog2e, (E*)o, ldo));                                                                     \
    return EFQAT_OK;                                                                                                               \
  } while (0)
  if (dtype == EFQAT_F32) { if (dim <= 64) EFQAT_DEC(float, 64); if (dim <= 96) EFQAT_DEC(float, 96); EFQAT_DEC(float, 128); }
  if (dim <= 64) EFQAT_DEC(bf16_t, 64);
  if (dim <= 96) EFQAT_DEC(bf16_t, 96);
  EFQAT_DEC(bf16_t, 128);
#undef EFQAT_DEC
}
