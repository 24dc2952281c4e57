// Attention of one new token per sequence where the sequences share a prefix:
//   out[b][h] = sum_j softmax_j(scale q[b][h] . K_j) V_j,
// j over the shared tokens (one block table for all) and then the sequence's own.
//
// The queries of all sequences and of one key head are the rows of one product with
// the prefix's keys, up to 64 at a time, so that a shared key is read once for 64
// queries.  A workgroup takes a run of the prefix's keys for its rows, a wave one of a
// sequence's own tokens; either keeps the running maximum m, sum l of exp2(score - m) and
// value sum O, and leaves them as a part in the workspace; a second kernel joins the
// parts of each query.  Both kinds of run are in one launch, so that a CU has some of
// each: the prefix's are bound by their instructions, the own tokens' by what one
// CU reads (32 query and 8 key heads of 128, bf16, us with the join: 64 sequences of up to
// 512 own tokens behind 8192 shared 44, without the prefix 20.4, without own tokens 40 at
// one workgroup a CU; 16 behind 2000 15; 2 of 40 behind 501 9).  A step of 64 shared keys
// and 64 rows takes 4600 cycles, of which 1000 are matrix products, 1800 with the reads
// and turns of the values, 1300 the loads and the scores, 600 the exponents, 900 the
// stores and barriers, one after the other in the one wave of the prefix that a SIMD has;
// the registers hold one more, which has own tokens.  Own tokens by whole workgroups, four
// waves to a run, joined in LDS, took 23.3 us for 20.4, and 52 for 32 where many have few
// (114 sequences of up to 39, 64 and 8 heads of 256).
//
// As in the attention of single sequences,
//   S (keys x queries) = K Q^T,   O^T (values x queries) = V^T P^T
// leave one query in lane column l % 16, and the second product takes its keys in the
// order in which the first left them: no exchange between the products.
#include "attn_tile.h"

namespace d2moe {
namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr int kRows = 16;  // queries of a lane column set
// How far (in units of log2) scores may lie above the reference that they are weighed
// by: it is the largest score when it is set, and moves only past this, so that most
// tiles neither look for the largest among lanes nor rescale the value sums.
constexpr float kRoom = 8.0f;
constexpr int kSpan = 512;  // keys whose row offsets are worked out at a time

struct PrefixArgs {
  const void *q, *k, *v;
  int64_t q_stride, page_stride, token_stride, head_stride;
  const int32_t *table, *lengths, *prefix_table, *prefix_lens;
  FastDiv page, per_head, by_heads, by_tiles, by_head_tiles, by_seqs;  // (per_head: by G)
  int B, n_pages, max_pages, prefix_pages, Hq, H, G, D;
  float scale_log2;  // scale / ln 2
  int row_tiles, splits, chunk;           // of the prefix: row tiles, runs of `chunk` keys
  int head_tiles, own_splits, own_chunk;  // of a sequence's own tokens
  int shared_groups, own_runs;
  float *shared_o, *shared_ml, *own_o, *own_ml;  // parts: rows of D and of (m, l)
  void* out;
};

// Tokens of sequence b that lie in the prefix, and the end of its own.
__device__ inline int shared_end(const PrefixArgs& a, int b) {
  const int64_t room = (int64_t)a.prefix_pages * a.page.d;
  int p = a.prefix_lens[b];
  const int n = a.lengths[b];
  p = p < n ? p : n;
  return p < 0 ? 0 : p > room ? (int)room : p;
}
__device__ inline int own_end(const PrefixArgs& a, int b) {
  const int64_t room = (int64_t)a.max_pages * a.page.d;
  const int n = a.lengths[b];
  return n < 0 ? 0 : n > room ? (int)room : n;
}

// The products of a wave: TK keys with 16 queries a column set.  K and V lie in LDS as
// rows of CPR chunks of 16 bytes, K's swizzled.  Of a value row a lane takes VE
// consecutive values, 16 lanes a run of 16 VE; element i of run h is row l % 16 of value
// product (h, i).
template <typename T, int DP>
struct Products;

template <int DP>
struct Products<uint16_t, DP> {
  static constexpr int TK = 32, PER = 8, CPR = DP / PER, KS = CPR / 4;
  static constexpr int VE = DP >= 128 ? 8 : 4, H = DP / (16 * VE), NS = 8;
  struct Q { u4 f[KS]; };
  __device__ static int key_of(int j, int q) { return j < 4 ? 4 * q + j : 12 + 4 * q + j; }
  __device__ static void load_q(Q& o, const uint16_t* row, int q, int D) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 32 * s + 8 * q;
      o.f[s] = row && c < D ? *(const u4*)(row + c) : u4{0, 0, 0, 0};
    }
  }
  // key(t, c): chunk 4 c + lane / 16 of row 16 t + lane % 16
  template <int CT, typename Key>
  __device__ static void scores(f4 (&s)[CT][2], Key key, const Q (&q)[CT]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      u4 x[KS];
#pragma unroll
      for (int c = 0; c < KS; ++c) x[c] = key(t, c);
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) {
        s[ct][t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < KS; ++c) s[ct][t] = mma(x[c], q[ct].f[c], s[ct][t]);
      }
    }
  }
  // p as three bf16 pieces whose sum is exact: each is what is left, rounded, and leaves
  // eight bits less.
  struct P { u4 piece[3]; };
  __device__ static void split(P& o, const float (&p)[NS]) {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      float a = p[2 * d], b = p[2 * d + 1];
#pragma unroll
      for (int k = 0; k < 3; ++k) {
        const uint32_t both = pack(a, b);
        o.piece[k][d] = both;
        if (k < 2) {
          a -= __uint_as_float(both << 16);
          b -= __uint_as_float(both & 0xffff0000u);
        }
      }
    }
  }
  __device__ static uint32_t pack(float a, float b) {  // to nearest even
    typedef float f2 __attribute__((ext_vector_type(2)));
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
  }
  // value(j, h): the VE values of row key_of(j) from 16 VE h + VE (lane % 16) on
  typedef uint32_t V __attribute__((ext_vector_type(VE / 2)));
  template <int CT, typename Value>
  __device__ static void values(f4 (&o)[CT][H][VE], const P (&p)[CT], Value value) {
#pragma unroll
    for (int h = 0; h < H; ++h) {
      V x[NS];
#pragma unroll
      for (int j = 0; j < NS; ++j) x[j] = value(j, h);
      // four elements at a time, so that no product waits for the one before it
#pragma unroll
      for (int i0 = 0; i0 < VE; i0 += 4) {
        u4 a[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int d = 0; d < 4; ++d)
            a[i][d] = __builtin_amdgcn_perm(x[2 * d + 1][(i0 + i) / 2], x[2 * d][(i0 + i) / 2],
                                            (i & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
              o[ct][h][i0 + i] = mma(a[i], p[ct].piece[k], o[ct][h][i0 + i]);
      }
    }
  }
};

template <int DP>
struct Products<float, DP> {
  static constexpr int TK = 16, PER = 4, CPR = DP / PER, KS = CPR / 4;
  static constexpr int VE = 4, H = DP / 64, NS = 4;
  struct Q { f4 f[KS]; };
  __device__ static int key_of(int j, int q) { return 4 * q + j; }
  __device__ static void load_q(Q& o, const float* row, int q, int D) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 16 * s + 4 * q;
      o.f[s] = row && c < D ? *(const f4*)(row + c) : f4{0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
  template <int CT, typename Key>
  __device__ static void scores(f4 (&s)[CT][1], Key key, const Q (&q)[CT]) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) s[ct][0] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      const f4 x = __builtin_bit_cast(f4, key(0, c));
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          const f4 acc = s[ct][0];
          s[ct][0] = mma(x[e], q[ct].f[c][e], acc);
          // nor shares part of its registers with the sum so far
          if (c + e > 0) asm("" : "+v"(s[ct][0]) : "v"(acc));
        }
    }
  }
  struct P { float p[NS]; };
  __device__ static void split(P& o, const float (&p)[NS]) {
#pragma unroll
    for (int j = 0; j < NS; ++j) o.p[j] = p[j];
  }
  typedef u4 V;
  template <int CT, typename Value>
  __device__ static void values(f4 (&o)[CT][H][VE], const P (&p)[CT], Value value) {
#pragma unroll
    for (int j = 0; j < NS; ++j)
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const f4 x = __builtin_bit_cast(f4, value(j, h));
#pragma unroll
        for (int i = 0; i < VE; ++i)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) o[ct][h][i] = mma(x[i], p[ct].p[j], o[ct][h][i]);
      }
  }
};

// A tile's scores to the weights of its values: in units of log2, less the reference m;
// above kRoom the reference moves, and l and o with it.  Where `masks`, masked(ct, key)
// says which of a lane's are none.
template <typename M, int CT, typename Masked>
__device__ inline void weigh(typename M::P (&p)[CT], const f4 (&sc)[CT][M::NS / 4], float scale,
                             float (&m)[CT], float (&l)[CT], f4 (&o)[CT][M::H][M::VE], bool masks,
                             Masked masked, int q) {
  float x[CT][M::NS], mx[CT];
  bool moves = false;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const float ref = m[ct] == -INFINITY ? 0.0f : m[ct];
#pragma unroll
    for (int j = 0; j < M::NS; ++j) x[ct][j] = fmaf(sc[ct][j / 4][j % 4], scale, -ref);
  }
  if (masks) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int j = 0; j < M::NS; ++j)
        if (masked(ct, M::key_of(j, q))) x[ct][j] = -INFINITY;
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    mx[ct] = -INFINITY;
#pragma unroll
    for (int j = 0; j < M::NS; ++j) mx[ct] = fmaxf(mx[ct], x[ct][j]);
    moves |= mx[ct] > (m[ct] == -INFINITY ? -INFINITY : kRoom);
  }
  if (__any(moves)) {
#pragma unroll
    for (int ct = 0; ct < CT; ++ct) {
      mx[ct] = fmaxf(mx[ct], __shfl_xor(mx[ct], 16, 64));
      mx[ct] = fmaxf(mx[ct], __shfl_xor(mx[ct], 32, 64));
      // the largest score so far, where there is one
      const float ref = m[ct] == -INFINITY ? 0.0f : m[ct], top = fmaxf(m[ct], ref + mx[ct]);
      const float by = top == -INFINITY ? 0.0f : top - ref, alpha = fast_exp2(m[ct] - ref - by);
      m[ct] = top;
      l[ct] *= alpha;
#pragma unroll
      for (int j = 0; j < M::NS; ++j) x[ct][j] -= by;
#pragma unroll
      for (int h = 0; h < M::H; ++h)
#pragma unroll
        for (int i = 0; i < M::VE; ++i) o[ct][h][i] *= alpha;
    }
  }
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
    for (int j = 0; j < M::NS; ++j) {
      x[ct][j] = fast_exp2(x[ct][j]);
      l[ct] += x[ct][j];
    }
    M::split(p[ct], x[ct]);
  }
}

// A run's division among the waves: NC of them share a tile of keys, CT column sets
// each, the others (kWaves / NC key groups) take other tiles of the same step.
template <typename T, int DP, int CT, int NC>
struct Run {
  using M = Products<T, DP>;
  static constexpr int NG = kWaves / NC, KEYS = NG * M::TK, ROWS = 16 * CT * NC;
  static constexpr int EACH = KEYS * M::CPR / kThreads;  // chunks of K, and of V, a thread
  static_assert(KEYS * M::CPR % kThreads == 0, "whole chunks");
  static_assert(kSpan % KEYS == 0, "whole steps");
  struct Step {
    int64_t off[2][kSpan];  // of the keys' rows, -1 where there is none: spans in turn
    u4 k[KEYS * M::CPR], v[KEYS * M::CPR];
  };
  struct Join {
    float m[NG][ROWS], l[NG][ROWS];
    __align__(16) float o[NG][ROWS][DP + 4];
  };
  union Lds {
    Step step;
    Join join;
  };
};

// One row's value sum by a wave, a key after the other and only those that it attends.  In
// the matrix products 0 times an infinite or NaN value is not 0, so that such a value
// reaches the rows of a tile that do not attend its key as well: seldom, and their sums are
// made here once more (64 sequences behind 8192 tokens, a fourth of them sharing 4000, with
// an infinite value further on: 47.2 us, without one 43.3).
__device__ inline float value_of(const uint16_t* p) { return bf2f(*p); }
__device__ inline float value_of(const float* p) { return *p; }
template <typename T, int DP>
__device__ void own_sum(const PrefixArgs& a, const int32_t* table, const T* kc, const T* vc,
                        const T* query, int k0, int k1, float m, float* out) {
  constexpr int N = DP / 64;  // dimensions of a lane
  const int lane = threadIdx.x & 63;
  float q[N], sum[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    sum[i] = 0.0f;
    q[i] = 64 * i + lane < a.D ? value_of(query + 64 * i + lane) : 0.0f;
  }
#pragma unroll 1
  for (int key = k0; key < k1; ++key) {
    const uint32_t at = a.page.div(key);
    const int page = table[at];
    if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
    const int64_t off = page * a.page_stride + (int64_t)(key - at * a.page.d) * a.token_stride;
    float score = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (64 * i + lane < a.D) score = fmaf(q[i], value_of(kc + off + 64 * i + lane), score);
#pragma unroll
    for (int by = 1; by < 64; by *= 2) score += __shfl_xor(score, by, 64);
    const float w = fast_exp2(fmaf(score, a.scale_log2, -m));
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (64 * i + lane < a.D) sum[i] = fmaf(w, value_of(vc + off + 64 * i + lane), sum[i]);
  }
#pragma unroll
  for (int i = 0; i < N; ++i)
    if (64 * i + lane < a.D) out[64 * i + lane] = sum[i];
}

// Keys k0 .. k1 - 1 of `table` (pages of it) and key head hk for the rows of a tile:
// row(r) is query r, or null; limit(r) the end of the keys that it attends.  Rows 0 ..
// rows - 1 go to part_o and part_ml.
template <typename T, int DP, int CT, int NC, typename RowOf, typename LimitOf>
__device__ void attend(const PrefixArgs& a, typename Run<T, DP, CT, NC>::Lds& lds,
                       const int32_t* table, int pages, int hk, int k0, int k1, RowOf row_of,
                       LimitOf limit_of, int rows, float* part_o, float* part_ml) {
  using R = Run<T, DP, CT, NC>;
  using M = typename R::M;
  constexpr int CPR = M::CPR, PER = M::PER, EACH = R::EACH;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), kg = wave / NC, cg = wave % NC;
  if (k1 <= k0) {
    if (tid < rows) *(float2*)(part_ml + 2 * tid) = make_float2(-INFINITY, 0.0f);
    return;
  }
  const T* kc = (const T*)a.k + hk * a.head_stride;
  const T* vc = (const T*)a.v + hk * a.head_stride;
  typename M::Q qf[CT];
  int limit[CT], least = 0x7fffffff;
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int r = (cg * CT + ct) * 16 + col;
    M::load_q(qf[ct], (const T*)row_of(r), q, a.D);
    limit[ct] = limit_of(r);
    least = limit[ct] < least ? limit[ct] : least;
  }
  float m[CT], l[CT];
  f4 o[CT][M::H][M::VE];
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    m[ct] = -INFINITY, l[ct] = 0.0f;
#pragma unroll
    for (int h = 0; h < M::H; ++h)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) o[ct][h][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // Row offsets by all threads, a span at a time: written to LDS where the span before
  // it begins, their block-table entries read a span earlier.
  constexpr int kOwn = kSpan / kThreads, kPer = kSpan / R::KEYS;
  const int steps = (k1 - k0 + R::KEYS - 1) / R::KEYS, spans = (steps + kPer - 1) / kPer;
  int page[kOwn];
  auto fetch = [&](int span) {
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
      const uint32_t at = a.page.div(k0 + span * kSpan + e * kThreads + tid);
      page[e] = table[at < (uint32_t)pages ? at : (uint32_t)pages - 1];
    }
  };
  auto put = [&](int span) {
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
      const uint32_t key = k0 + span * kSpan + e * kThreads + tid;
      const bool in = key < (uint32_t)k1 && (uint32_t)page[e] < (uint32_t)a.n_pages;
      lds.step.off[span & 1][e * kThreads + tid] =
          in ? page[e] * a.page_stride +
                   (int64_t)(key - a.page.div(key) * a.page.d) * a.token_stride
             : -1;
    }
  };
  // chunk e of this thread: row (e kThreads + tid) / CPR of the step, chunk tid % CPR;
  // chunks past the head's end are zero
  const int c = tid % CPR;
  const bool wide = c * PER < a.D;
  const T *kd = kc + c * PER, *vd = vc + c * PER;
  u4 kf[EACH], vf[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) kf[e] = vf[e] = u4{0, 0, 0, 0};
  uint32_t holes = 0;
  auto load = [&](int s) {  // whatever row where there is no key
    const int64_t* off = lds.step.off[s / kPer & 1] + s % kPer * R::KEYS;
    holes = 0;
    int64_t at[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) at[e] = off[(e * kThreads + tid) / CPR];
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      holes |= (at[e] < 0 ? 1u : 0u) << e;
      at[e] = at[e] < 0 ? 0 : at[e];
    }
    if (wide) {
#pragma unroll
      for (int e = 0; e < EACH; ++e) kf[e] = *(const u4*)(kd + at[e]);
#pragma unroll
      for (int e = 0; e < EACH; ++e) vf[e] = *(const u4*)(vd + at[e]);
    }
  };
  fetch(0);
  put(0);
  if (spans > 1) fetch(1);
  lds_barrier();
  load(0);
  for (int s = 0; s < steps; ++s) {
    lds_barrier();  // the step before has been used
    if (__any(holes)) {  // 0 times what a masked row holds is not 0
#pragma unroll
      for (int e = 0; e < EACH; ++e)
        if (holes >> e & 1) vf[e] = u4{0, 0, 0, 0};
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int row = (e * kThreads + tid) / CPR;
      lds.step.k[row * CPR + (c ^ swizzle<CPR>(row))] = kf[e];
      lds.step.v[row * CPR + c] = vf[e];
    }
    const int span = s / kPer;
    if (s % kPer == 0 && span + 1 < spans) put(span + 1);
    lds_barrier();
    if (s + 1 < steps) load(s + 1);
    if (s % kPer == 0 && span + 2 < spans) fetch(span + 2);

    // the keys of this wave's tile that are none
    const uint32_t none = (uint32_t)__ballot(
        lds.step.off[span & 1][s % kPer * R::KEYS + kg * M::TK + (lane & (M::TK - 1))] < 0);
    f4 sc[CT][M::NS / 4];
    const u4* kt = lds.step.k + kg * M::TK * CPR;
    M::scores(sc, [&](int t, int c) {
      const int row = 16 * t + col;
      return kt[row * CPR + ((4 * c + q) ^ swizzle<CPR>(row))];
    }, qf);
    const int first = k0 + s * R::KEYS + kg * M::TK;
    const bool border = __any(first + M::TK > least);
    typename M::P p[CT];
    weigh<M>(p, sc, a.scale_log2, m, l, o, none != 0 || border, [&](int ct, int key) {
      return (none >> key & 1) || first + key >= limit[ct];
    }, q);
    const u4* vt = lds.step.v + kg * M::TK * CPR;
    M::values(o, p, [&](int j, int h) {
      return ((const typename M::V*)(vt + M::key_of(j, q) * CPR))[16 * h + col];
    });
  }

  // join the key groups: every row's m, l and O
  lds_barrier();
#pragma unroll
  for (int ct = 0; ct < CT; ++ct) {
    const int r = (cg * CT + ct) * 16 + col;
    l[ct] += __shfl_xor(l[ct], 16, 64);
    l[ct] += __shfl_xor(l[ct], 32, 64);
    if (q == 0) {
      lds.join.m[kg][r] = m[ct];
      lds.join.l[kg][r] = l[ct];
    }
#pragma unroll
    for (int h = 0; h < M::H; ++h)
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < M::VE; i += 4)
          *(f4*)&lds.join.o[kg][r][16 * M::VE * h + M::VE * (4 * q + e) + i] =
              f4{o[ct][h][i][e], o[ct][h][i + 1][e], o[ct][h][i + 2][e], o[ct][h][i + 3][e]};
  }
  lds_barrier();
  if (tid < R::ROWS) {  // the groups' factors, in the place of m
    float mm = -INFINITY, ll = 0.0f;
#pragma unroll
    for (int g = 0; g < R::NG; ++g) mm = fmaxf(mm, lds.join.m[g][tid]);
    const float ref = mm == -INFINITY ? 0.0f : mm;
#pragma unroll
    for (int g = 0; g < R::NG; ++g) {
      const float f = fast_exp2(lds.join.m[g][tid] - ref);
      ll = fmaf(f, lds.join.l[g][tid], ll);
      lds.join.m[g][tid] = f;
    }
    if (tid < rows) *(float2*)(part_ml + 2 * tid) = make_float2(mm, ll);
    lds.join.l[0][tid] = mm;
  }
  __shared__ int spoilt;  // whether a sum is not finite
  if (tid == 0) spoilt = 0;
  lds_barrier();
  constexpr int kRow = DP / 4;  // threads of a row
  const int d = tid % kRow * 4;
  float zero = 0.0f;  // as long as the sums are finite
  if (d < a.D)
    for (int r = tid / kRow; r < rows; r += kThreads / kRow) {
      f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int g = 0; g < R::NG; ++g) acc += lds.join.m[g][r] * *(const f4*)&lds.join.o[g][r][d];
      *(f4*)(part_o + (int64_t)r * a.D + d) = acc;
      zero = fmaf(0.0f, acc[0] + acc[1] + acc[2] + acc[3], zero);
    }
  if (zero != 0.0f) spoilt = 1;
  lds_barrier();
  if (spoilt == 0) return;
  __syncthreads();  // the sums to be replaced have been written
  for (int r = wave; r < rows; r += kWaves) {
    const int end = limit_of(r);
    if (end < k1)  // (what a row attends whole is its own)
      own_sum<T, DP>(a, table, kc, vc, row_of(r), k0, end, lds.join.l[0][r],
                     part_o + (int64_t)r * a.D);
  }
}

// Row tiles of the prefix, 16 CT NC rows each: query r of a key head is head r % G of
// sequence r / G.
template <typename T, int DP, int CT, int NC>
__device__ void attend_shared(const PrefixArgs& a, typename Run<T, DP, CT, NC>::Lds& lds, int u) {
  constexpr int ROWS = Run<T, DP, CT, NC>::ROWS;
  const int v = a.by_heads.div(u), hk = u - v * a.H;
  const int split = a.by_tiles.div(v), tile = v - split * a.row_tiles;
  const int r0 = tile * ROWS, total = a.B * a.G, rows = total - r0 < ROWS ? total - r0 : ROWS;
  // the end of the keys that any row attends
  __shared__ int last;
  if (threadIdx.x < 64) {  // (ROWS <= 64)
    int n = (int)threadIdx.x < rows ? shared_end(a, a.per_head.div(r0 + threadIdx.x)) : 0;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
      const int other = __shfl_xor(n, off, 64);
      n = other > n ? other : n;
    }
    if (threadIdx.x == 0) last = n;
  }
  lds_barrier();
  const int k0 = split * a.chunk;
  const int end = last, k1 = split + 1 < a.splits && k0 + a.chunk < end ? k0 + a.chunk : end;
  const int64_t part = (int64_t)u * ROWS;
  attend<T, DP, CT, NC>(
      a, lds, a.prefix_table, a.prefix_pages, hk, k0, k1,
      [&](int r) -> const T* {
        if (r >= rows) return nullptr;
        const int b = a.per_head.div(r0 + r), g = r0 + r - b * a.G;
        return (const T*)a.q + b * a.q_stride + (int64_t)(hk * a.G + g) * a.D;
      },
      [&](int r) { return r < rows ? shared_end(a, a.per_head.div(r0 + r)) : 0x7fffffff; }, rows,
      a.shared_o + part * a.D, a.shared_ml + part * 2);
}

// A run of a sequence's own tokens by one wave, up to 16 query heads of a key head, which
// waits for no other: tiles of TK keys, keys through LDS for whole rows' loads, values from
// memory to the products' registers, the next tile's while this one is weighed.  Row offsets
// go through LDS a tile ahead, their block-table entries two.
template <typename T, int DP>
struct OwnLds {
  int64_t off[2][Products<T, DP>::TK];
  u4 k[Products<T, DP>::TK * Products<T, DP>::CPR];
};
template <typename T, int DP>
__device__ void attend_own(const PrefixArgs& a, OwnLds<T, DP>& lds, int u) {
  using M = Products<T, DP>;
  constexpr int TK = M::TK, CPR = M::CPR, EACH = TK * CPR / 64;
  const int lane = threadIdx.x & 63, col = lane & 15, q = lane >> 4;
  const int x = a.by_heads.div(u), hk = u - x * a.H;
  const int w = a.by_head_tiles.div(x), tile = x - w * a.head_tiles;
  const int split = a.by_seqs.div(w), b = w - split * a.B;
  const int g0 = tile * kRows, rows = a.G - g0 < kRows ? a.G - g0 : kRows;
  const int64_t part = (int64_t)u * (a.G < kRows ? a.G : kRows);
  float* part_ml = a.own_ml + part * 2;
  const int from = shared_end(a, b), end = own_end(a, b);
  const int64_t first = from + (int64_t)split * a.own_chunk;
  const int k1 = split + 1 < a.own_splits && first + a.own_chunk < end ? (int)first + a.own_chunk
                                                                       : end;
  if (k1 <= first) {
    if (lane < rows) *(float2*)(part_ml + 2 * lane) = make_float2(-INFINITY, 0.0f);
    return;
  }
  const int k0 = (int)first, tiles = (k1 - k0 + TK - 1) / TK;
  const int32_t* table = a.table + (int64_t)b * a.max_pages;
  const T* kc = (const T*)a.k + hk * a.head_stride;
  const T* vc = (const T*)a.v + hk * a.head_stride;
  int page;
  auto fetch = [&](int t) {
    const uint32_t at = a.page.div(k0 + t * TK + (lane & (TK - 1)));
    page = table[at < (uint32_t)a.max_pages ? at : (uint32_t)a.max_pages - 1];
  };
  auto put = [&](int t) {  // returns which are none
    const uint32_t key = k0 + t * TK + (lane & (TK - 1));
    const bool in = key < (uint32_t)k1 && (uint32_t)page < (uint32_t)a.n_pages;
    if (lane < TK)
      lds.off[t & 1][lane] = in ? page * a.page_stride +
                                  (int64_t)(key - a.page.div(key) * a.page.d) * a.token_stride
                            : 0;  // whatever row where there is no key
    return (uint32_t)__ballot(!in);
  };
  fetch(0);
  typename M::Q qf[1];
  M::load_q(qf[0],
            col < rows ? (const T*)a.q + b * a.q_stride + (int64_t)(hk * a.G + g0 + col) * a.D
                       : nullptr,
            q, a.D);
  // chunk e of this lane: row (64 e + lane) / CPR of the tile, chunk lane % CPR; chunks
  // past the head's end are zero
  const int c = lane % CPR;
  const bool wide = c * M::PER < a.D;
  u4 kf[EACH];
  typename M::V vf[M::NS][M::H];
#pragma unroll
  for (int e = 0; e < EACH; ++e) kf[e] = u4{0, 0, 0, 0};
  auto load_k = [&](int t) {
    int64_t at[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) at[e] = lds.off[t & 1][(64 * e + lane) / CPR] + c * M::PER;
    if (wide) {
#pragma unroll
      for (int e = 0; e < EACH; ++e) kf[e] = *(const u4*)(kc + at[e]);
    }
  };
  auto load_v = [&](int t) {
#pragma unroll
    for (int j = 0; j < M::NS; ++j) {
      const T* row = vc + lds.off[t & 1][M::key_of(j, q)];
#pragma unroll
      for (int h = 0; h < M::H; ++h) {  // (products past the head's end are not used)
        const int d = M::VE * (16 * h + col);
        vf[j][h] = *(const typename M::V*)(row + (d < a.D ? d : 0));
      }
    }
  };
  uint32_t none = put(0);
  if (tiles > 1) fetch(1);
  wave_handoff();
  load_k(0);
  load_v(0);
  float m[1] = {-INFINITY}, l[1] = {0.0f};
  f4 o[1][M::H][M::VE];
#pragma unroll
  for (int h = 0; h < M::H; ++h)
#pragma unroll
    for (int i = 0; i < M::VE; ++i) o[0][h][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int t = 0; t < tiles; ++t) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int row = (64 * e + lane) / CPR;
      lds.k[row * CPR + (c ^ swizzle<CPR>(row))] = kf[e];
    }
    const uint32_t now = none;
    if (t + 1 < tiles) none = put(t + 1);
    wave_handoff();
    if (t + 1 < tiles) load_k(t + 1);
    if (t + 2 < tiles) fetch(t + 2);
    f4 sc[1][M::NS / 4];
    M::scores(sc, [&](int i, int x) {
      const int row = 16 * i + col;
      return lds.k[row * CPR + ((4 * x + q) ^ swizzle<CPR>(row))];
    }, qf);
    wave_handoff();  // the tile's keys have been read
    typename M::P p[1];
    weigh<M>(p, sc, a.scale_log2, m, l, o, now != 0,
             [&](int, int key) { return now >> key & 1; }, q);
    if (now != 0) {  // 0 times what a masked row holds is not 0
#pragma unroll
      for (int j = 0; j < M::NS; ++j)
        if (now >> M::key_of(j, q) & 1)
#pragma unroll
          for (int h = 0; h < M::H; ++h) vf[j][h] = typename M::V{};
    }
    M::values(o, p, [&](int j, int h) { return vf[j][h]; });
    if (t + 1 < tiles) load_v(t + 1);
  }
  l[0] += __shfl_xor(l[0], 16, 64);
  l[0] += __shfl_xor(l[0], 32, 64);
  if (col >= rows) return;
  if (q == 0) *(float2*)(part_ml + 2 * col) = make_float2(m[0], l[0]);
  float* row = a.own_o + (part + col) * a.D;
#pragma unroll
  for (int h = 0; h < M::H; ++h)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int i = 0; i < M::VE; i += 4) {
        const int d = 16 * M::VE * h + M::VE * (4 * q + e) + i;
        if (d < a.D)
          *(f4*)(row + d) = f4{o[0][h][i][e], o[0][h][i + 1][e], o[0][h][i + 2][e],
                               o[0][h][i + 3][e]};
      }
}

// The prefix's workgroups, which take longest, then the own tokens'.
template <typename T, int DP, int CT, int NC>
__global__ __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) void attn_prefix_kernel(PrefixArgs a) {
  union Lds {
    typename Run<T, DP, CT, NC>::Lds shared;
    OwnLds<T, DP> own[kWaves];
  };
  __shared__ Lds lds;
  if ((int)blockIdx.x < a.shared_groups) {
    attend_shared<T, DP, CT, NC>(a, lds.shared, blockIdx.x);
  } else {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int u = (blockIdx.x - a.shared_groups) * kWaves + wave;
    if (u < a.own_runs) attend_own<T, DP>(a, lds.own[wave], u);
  }
}

// Joins the parts of a query, a workgroup each: the prefix's runs, then its own, one
// after the other by parts of a wave (half a wave has 128 values), four of them loaded
// together.
template <typename T, int LANES>
__global__ __launch_bounds__(kThreads) void attn_prefix_join_kernel(PrefixArgs a, int tile_rows) {
  constexpr int kSubs = kThreads / LANES, kAhead = 4;
  __shared__ float pm[kSubs], pl[kSubs];
  __shared__ __align__(16) f4 po[kSubs][LANES];
  const int head = blockIdx.x, b = blockIdx.y;
  const int hk = head / a.G, g = head - hk * a.G;
  const int sub = threadIdx.x / LANES, lane = threadIdx.x % LANES;
  const int d = 4 * lane < a.D ? 4 * lane : 0;
  const int own_rows = a.G < kRows ? a.G : kRows;
  const int r = b * a.G + g, tile = r / tile_rows, n = a.splits + a.own_splits;
  float mm = -INFINITY, ll = 0.0f;
  f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i0 = sub; i0 < n; i0 += kAhead * kSubs) {
    float2 ml[kAhead];
    f4 v[kAhead];
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      const int i = i0 + e * kSubs < n ? i0 + e * kSubs : i0;
      const float *o, *m;
      if (i < a.splits) {
        const int64_t p =
            (((int64_t)i * a.row_tiles + tile) * a.H + hk) * tile_rows + r % tile_rows;
        o = a.shared_o + p * a.D, m = a.shared_ml + p * 2;
      } else {
        const int64_t w = ((int64_t)(i - a.splits) * a.B + b) * a.head_tiles + g / kRows;
        const int64_t u = w * a.H + hk;
        const int64_t p = u * own_rows + g % kRows;
        o = a.own_o + p * a.D, m = a.own_ml + p * 2;
      }
      ml[e] = *(const float2*)m;
      v[e] = *(const f4*)(o + d);
    }
    float top = mm;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) top = fmaxf(top, ml[e].x);
    const float was = fast_exp2(mm - (top == -INFINITY ? 0.0f : top));
    mm = top;
    ll *= was;
    acc *= was;
#pragma unroll
    for (int e = 0; e < kAhead; ++e) {
      // without a key there may be no values written; scores that are NaN, which no maximum
      // knows of, have left a sum that is
      if (i0 + e * kSubs >= n || (ml[e].x == -INFINITY && ml[e].y == 0.0f)) continue;
      const float f = fast_exp2(ml[e].x - mm);
      ll = fmaf(f, ml[e].y, ll);
      acc += f * v[e];
    }
  }
  po[sub][lane] = acc;
  if (lane == 0) pm[sub] = mm, pl[sub] = ll;
  __syncthreads();
  if (sub != 0 || 4 * lane >= a.D) return;
#pragma unroll
  for (int i = 1; i < kSubs; ++i) mm = fmaxf(mm, pm[i]);
  const float ref = mm == -INFINITY ? 0.0f : mm;
  ll = 0.0f;
  acc = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kSubs; ++i) {
    const float f = fast_exp2(pm[i] - ref);
    ll = fmaf(f, pl[i], ll);
    acc += f * po[i][lane];
  }
  store4((T*)a.out + ((int64_t)b * a.Hq + head) * a.D + d,
         acc * (ll == 0.0f ? 0.0f : 1.0f / ll));
}

// How a call is divided, from the sizes alone.
struct Plan {
  int tile_rows, row_tiles, splits, chunk, head_tiles, own_splits, own_chunk;
};
// Runs that the keys are cut into: of the prefix's one a CU (64 sequences behind 8192
// keys 44 us, with 128 of them 64, with 512 48; the other way without own tokens, 40 and
// 36; 129 to 255 units are one run each, which leaves CUs without one), of the own tokens
// eight a CU (64 sequences of up to 512, 12 heads of 64 in fp32: 30.0 us, with 1024 of them
// 37.4; 4096 take 22.7 for 20.4 with 32 and 8 heads of 128 in bf16); and the least keys of a
// run (of the prefix: 16 sequences behind 2000 15.6 us, with 64 19.1, with 256 16.6; of the
// own tokens: 9 of 300 behind 1500, fp32, 10.9 us, with 128 13.9; 32 of 300 with heads of
// 256 47.5, with 32 53.6).
constexpr int kSharedGroups = 256, kOwnRuns = 2048;
constexpr int kLeastKeys = 128, kLeastOwn = 64;
constexpr int kMostSplits = 64;

void divide(int keys, int64_t units, int groups, int least, int& splits, int& chunk) {
  int64_t most = units >= groups ? 1 : groups / units;
  most = most < kMostSplits ? most : kMostSplits;
  const int64_t need = ((int64_t)keys + least - 1) / least;
  splits = (int)(need < most ? need : most);
  if (splits < 1) splits = 1;
  chunk = (int)(((int64_t)keys + splits - 1) / splits + 31) / 32 * 32;
  if (chunk < least) chunk = least;
}

// No fewer runs than divide() makes of this many units or fewer: fewer units are cut into
// more runs each, and a workspace for the largest batch is to serve every smaller one.
int64_t most_runs(int keys, int64_t units, int groups, int least) {
  int64_t splits = ((int64_t)keys + least - 1) / least;
  splits = splits < 1 ? 1 : splits < kMostSplits ? splits : kMostSplits;
  const int64_t runs = units * splits < groups ? units * splits : groups;
  return runs > units ? runs : units;
}

Plan plan_of(int B, int q_heads, int n_heads, int max_prefix, int max_rest) {
  Plan p;
  const int G = q_heads / n_heads, rows = B * G;
  p.tile_rows = rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
  p.row_tiles = (rows + p.tile_rows - 1) / p.tile_rows;
  p.head_tiles = (G + kRows - 1) / kRows;
  divide(max_prefix, (int64_t)n_heads * p.row_tiles, kSharedGroups, kLeastKeys, p.splits, p.chunk);
  divide(max_rest, (int64_t)n_heads * p.head_tiles * B, kOwnRuns, kLeastOwn, p.own_splits,
         p.own_chunk);
  return p;
}
int64_t shared_rows(const Plan& p, int n_heads) {
  return (int64_t)n_heads * p.row_tiles * p.splits * p.tile_rows;
}
int64_t own_rows(const Plan& p, int B, int q_heads, int n_heads) {
  const int G = q_heads / n_heads;
  return (int64_t)n_heads * p.head_tiles * B * p.own_splits * (G < kRows ? G : kRows);
}

template <typename T, int DP>
hipError_t run_prefix_d(const PrefixArgs& a, int tile_rows, hipStream_t s) {
  const int grid = a.shared_groups + (a.own_runs + kWaves - 1) / kWaves;
  if (tile_rows == 16)
    attn_prefix_kernel<T, DP, 1, 1><<<grid, kThreads, 0, s>>>(a);
  else if (tile_rows == 32)
    attn_prefix_kernel<T, DP, 1, 2><<<grid, kThreads, 0, s>>>(a);
  else  // (wider rows leave no registers for two column sets)
    attn_prefix_kernel<T, DP, DP <= 128 ? 2 : 1, DP <= 128 ? 2 : 4><<<grid, kThreads, 0, s>>>(a);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  attn_prefix_join_kernel<T, DP <= 128 ? 32 : 64>
      <<<dim3(a.Hq, a.B), kThreads, 0, s>>>(a, tile_rows);
  return hipGetLastError();
}

template <typename T>
hipError_t run_prefix(const PrefixArgs& a, int tile_rows, hipStream_t s) {
  if (a.D <= 64) return run_prefix_d<T, 64>(a, tile_rows, s);
  if (a.D <= 128) return run_prefix_d<T, 128>(a, tile_rows, s);
  return run_prefix_d<T, 256>(a, tile_rows, s);
}

}  // namespace

size_t attn_prefix_workspace(int B, int q_heads, int n_heads, int dim, int max_prefix,
                             int max_rest) {
  if (B == 0) return 0;
  const Plan p = plan_of(B, q_heads, n_heads, max_prefix, max_rest);
  const int G = q_heads / n_heads;
  const int64_t tiles = (int64_t)n_heads * p.row_tiles;
  const int64_t own = (int64_t)n_heads * p.head_tiles * B;
  return (size_t)(most_runs(max_prefix, tiles, kSharedGroups, kLeastKeys) * p.tile_rows +
                  most_runs(max_rest, own, kOwnRuns, kLeastOwn) * (G < kRows ? G : kRows)) *
         (dim + 2) * sizeof(float);
}

hipError_t launch_attn_prefix(const void* q, int64_t q_stride, int B, int q_heads,
                              const d2moe_kv_cache* c, const int32_t* table, int max_pages,
                              const int32_t* lengths, const int32_t* prefix_table,
                              int prefix_pages, const int32_t* prefix_lens, int max_prefix,
                              int max_rest, float scale, void* out, void* ws, hipStream_t s) {
  if (B == 0) return hipSuccess;
  const Plan p = plan_of(B, q_heads, c->n_heads, max_prefix, max_rest);
  PrefixArgs a{};
  a.q = q, a.k = c->k, a.v = c->v, a.q_stride = q_stride, a.page_stride = c->page_stride;
  a.token_stride = c->token_stride, a.head_stride = c->head_stride;
  a.table = table, a.lengths = lengths, a.prefix_table = prefix_table;
  a.prefix_lens = prefix_lens, a.page = fast_div(c->page_size);
  a.per_head = fast_div(q_heads / c->n_heads), a.by_heads = fast_div(c->n_heads);
  a.B = B, a.n_pages = c->n_pages, a.max_pages = max_pages, a.prefix_pages = prefix_pages;
  a.Hq = q_heads, a.H = c->n_heads, a.G = q_heads / c->n_heads, a.D = c->head_dim;
  a.by_tiles = fast_div(p.row_tiles), a.by_head_tiles = fast_div(p.head_tiles);
  a.by_seqs = fast_div(B);
  a.scale_log2 = scale * kLog2e;
  a.row_tiles = p.row_tiles, a.splits = p.splits, a.chunk = p.chunk;
  a.head_tiles = p.head_tiles, a.own_splits = p.own_splits, a.own_chunk = p.own_chunk;
  a.shared_groups = c->n_heads * p.row_tiles * p.splits;
  a.own_runs = c->n_heads * p.head_tiles * B * p.own_splits;
  const int64_t rows = shared_rows(p, c->n_heads), own = own_rows(p, B, q_heads, c->n_heads);
  a.shared_o = (float*)ws, a.own_o = a.shared_o + rows * a.D;
  a.shared_ml = a.own_o + own * a.D, a.own_ml = a.shared_ml + rows * 2;
  a.out = out;
  return c->dtype == D2MOE_BF16 ? run_prefix<uint16_t>(a, p.tile_rows, s)
                                : run_prefix<float>(a, p.tile_rows, s);
}

}  // namespace d2moe
