// Attention of one new token per sequence over a paged key-value cache,
//   out[b][h] = sum_j softmax_j(scale q[b][h] . K_j) V_j,
// as one pass over the keys with the running maximum m, the sum l of
// exp(score - m) and the running value sum O, rescaled when m grows.
//
// The query heads of one key head (G of them, 16 at a time) are the columns of
// 16 x 16 matrix products, so a key or value row is read once for all of them:
//   S (keys x heads) = K Q^T,   O^T (values x heads) = V^T P^T.
// Both leave one head in lane column l % 16, and the four lanes of a column
// hold keys 4 q .. 4 q + 3 of a 16-key tile (q = l / 16).  The order of the
// keys in the second product is free, so its operand P^T takes exactly the
// keys that a lane computed, and V^T is read to match: no exchange between the
// products, only the maximum crosses lanes.
//
// The keys are split over workgroups (and their waves); splits leave their m, l
// and O in the workspace and a second kernel joins them.
//
// Bound by reading the cache: 4 len head_dim bytes (bf16) per key head against
// 16-column products that would take a twentieth of that time.
#include "decoder.h"

namespace d2moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kAttnWaves = 4;
constexpr int kAttnThreads = 64 * kAttnWaves;
constexpr int kHeadTile = 16;    // query heads of a workgroup
constexpr int kKeysAhead = 1024; // keys whose row offsets are held in LDS at a time
constexpr int kSplitUnit = 128;  // keys of a split are a multiple of this
constexpr int kSplitGroups = 2048;  // workgroups aimed at

struct AttnArgs {
  const void *q, *k, *v;
  int64_t q_stride, page_stride, token_stride, head_stride;
  const int32_t *table, *lengths;
  FastDiv page;
  int n_pages, max_pages, Hq, H, G, tiles, D, window, n_splits, chunk;
  float scale_log2;  // scale / ln 2
  void* out;
  float *part_o, *part_ml;  // [B][Hq][n_splits][D], [B][Hq][n_splits][2]
};

// Keys of sequence b that are attended: [first, first + count).
__device__ inline void key_range(const AttnArgs& a, int b, int& first, int& count) {
  int n = a.lengths[b];
  const int64_t room = (int64_t)a.max_pages * a.page.d;
  n = n < 0 ? 0 : n > room ? (int)room : n;
  first = a.window > 0 && n > a.window ? n - a.window : 0;
  count = n - first;
}

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline f4 mma(u4 a, u4 b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));  // the result gets registers of its own
  return d;
}
__device__ inline f4 mma(float a, float b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));
  return d;
}

// The tile products of one cache type: TK keys a step, a lane's share of the
// key rows (K), of the value rows (V) and of Q.  A lane loads VE consecutive
// values of a value row, dimensions 16 VE h + VE (l % 16) + 0 .. VE - 1, so that
// 16 lanes read a run of 16 VE values; element i of that run is the row l % 16
// of value product (h, i).  PAD: head_dim D is below DP; K and Q are zero past
// D, value loads past D read the row's start and their results are not used.
template <typename T, int DP, bool PAD>
struct Tile;

template <int DP, bool PAD>
struct Tile<uint16_t, DP, PAD> {
  static constexpr int TK = 32, VE = DP >= 128 ? 8 : 4, H = DP / (16 * VE), KS = DP / 32;
  static constexpr int NV = 8;  // value rows (keys) of a lane
  struct Q { u4 f[KS]; };
  struct K { u4 f[2][KS]; };
  struct V { uint32_t f[NV][H][VE / 2]; };

  __device__ static int key_of(int j, int q) { return j < 4 ? 4 * q + j : 12 + 4 * q + j; }

  __device__ static u4 chunk(const uint16_t* p, int c, int D) {
    if (PAD && c >= D) return u4{0, 0, 0, 0};
    return *(const u4*)(p + c);
  }
  __device__ static void load_q(Q& o, const uint16_t* row, int q, int D, bool live) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      o.f[s] = u4{0, 0, 0, 0};
      if (live) o.f[s] = chunk(row, 32 * s + 8 * q, D);
    }
  }
  __device__ static void load_k(K& o, const uint16_t* k, const int64_t* off, int lane, int D) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int64_t at = off[16 * t + (lane & 15)];
      const uint16_t* row = k + (at < 0 ? 0 : at);
#pragma unroll
      for (int s = 0; s < KS; ++s) o.f[t][s] = chunk(row, 32 * s + 8 * (lane >> 4), D);
    }
  }
  __device__ static void load_v(V& o, const uint16_t* v, const int64_t (&at)[NV], int lane, int D) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint16_t* row = v + (at[j] < 0 ? 0 : at[j]);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        int c = 16 * VE * h + VE * (lane & 15);
        if (PAD && c >= D) c = 0;
        if constexpr (VE == 8) {
          const u4 x = *(const u4*)(row + c);
#pragma unroll
          for (int d = 0; d < 4; ++d) o.f[j][h][d] = x[d];
        } else {
          const uint2 x = *(const uint2*)(row + c);
          o.f[j][h][0] = x.x;
          o.f[j][h][1] = x.y;
        }
      }
    }
  }
  __device__ static void clear_v(V& o, const int64_t (&at)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int d = 0; d < VE / 2; ++d) o.f[j][h][d] = at[j] < 0 ? 0u : o.f[j][h][d];
  }
  __device__ static void scores(float (&s)[NV], const K& k, const Q& q) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KS; ++c) acc = mma(k.f[t][c], q.f[c], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * t + i] = acc[i];
    }
  }
  // The probabilities enter as two bf16 terms: with one, its rounding (2^-8)
  // would be as large as that of the result; with two it is 2^-16.  The first
  // is cut, not rounded, and the second kept above zero, so that both have the
  // sign of the probability and an infinite value stays one.
  __device__ static void values(f4 (&o)[H][VE], const float (&p)[NV], const V& v) {
    u4 hi, lo;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      f2 rest;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        rest[e] = fmaxf(p[2 * d + e] -
                            __uint_as_float(__float_as_uint(p[2 * d + e]) & 0xffff0000u),
                        1.17549435e-38f);
      hi[d] = __builtin_amdgcn_perm(__float_as_uint(p[2 * d + 1]), __float_as_uint(p[2 * d]),
                                    0x07060302u);
      lo[d] = __builtin_bit_cast(uint32_t, __builtin_convertvector(rest, b2));
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        u4 a;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          a[d] = __builtin_amdgcn_perm(v.f[2 * d + 1][h][i / 2], v.f[2 * d][h][i / 2],
                                       (i & 1) ? 0x07060302u : 0x05040100u);
        o[h][i] = mma(a, hi, o[h][i]);
        o[h][i] = mma(a, lo, o[h][i]);
      }
  }
};

template <int DP, bool PAD>
struct Tile<float, DP, PAD> {
  static constexpr int TK = 16, VE = 4, H = DP / 64, KS = DP / 16;
  static constexpr int NV = 4;
  struct Q { f4 f[KS]; };
  struct K { f4 f[KS]; };
  struct V { f4 f[NV][H]; };

  __device__ static int key_of(int j, int q) { return 4 * q + j; }

  __device__ static f4 chunk(const float* p, int c, int D) {
    if (PAD && c >= D) return f4{0.0f, 0.0f, 0.0f, 0.0f};
    return *(const f4*)(p + c);
  }
  __device__ static void load_q(Q& o, const float* row, int q, int D, bool live) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      o.f[s] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      if (live) o.f[s] = chunk(row, 16 * s + 4 * q, D);
    }
  }
  __device__ static void load_k(K& o, const float* k, const int64_t* off, int lane, int D) {
    const int64_t at = off[lane & 15];
    const float* row = k + (at < 0 ? 0 : at);
#pragma unroll
    for (int s = 0; s < KS; ++s) o.f[s] = chunk(row, 16 * s + 4 * (lane >> 4), D);
  }
  __device__ static void load_v(V& o, const float* v, const int64_t (&at)[NV], int lane, int D) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const float* row = v + (at[j] < 0 ? 0 : at[j]);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        int c = 64 * h + 4 * (lane & 15);
        if (PAD && c >= D) c = 0;
        o.f[j][h] = *(const f4*)(row + c);
      }
    }
  }
  __device__ static void clear_v(V& o, const int64_t (&at)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) o.f[j][h][e] = at[j] < 0 ? 0.0f : o.f[j][h][e];
  }
  __device__ static void scores(float (&s)[NV], const K& k, const Q& q) {
    f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < KS; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc = mma(k.f[c][e], q.f[c][e], acc);
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = acc[i];
  }
  __device__ static void values(f4 (&o)[H][VE], const float (&p)[NV], const V& v) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < VE; ++i)
#pragma unroll
        for (int j = 0; j < NV; ++j) o[h][i] = mma(v.f[j][h][i], p[j], o[h][i]);
  }
};

template <typename T, int DP, bool PAD>
__global__ __launch_bounds__(kAttnThreads, 1) void attn_decode_kernel(AttnArgs a) {
  using M = Tile<T, DP, PAD>;
  constexpr int kPitch = DP + 4;
  __shared__ int64_t off[kKeysAhead];
  __shared__ float sm[kAttnWaves][kHeadTile], sl[kAttnWaves][kHeadTile];
  __shared__ __align__(16) float so[kAttnWaves][kHeadTile][kPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, col = lane & 15, q = lane >> 4;
  const int b = blockIdx.y;
  int unit = blockIdx.x;
  const int split = unit % a.n_splits;
  unit /= a.n_splits;
  const int hk = unit % a.H, tile = unit / a.H;
  int first, count;
  key_range(a, b, first, count);
  if (a.n_splits > 1 && (int64_t)split * a.chunk >= count) return;
  const int g0 = tile * kHeadTile;                               // of the key head's G heads
  const int heads = a.G - g0 < kHeadTile ? a.G - g0 : kHeadTile;  // of this workgroup
  const int h0 = hk * a.G + g0;
  const T* kc = (const T*)a.k + hk * a.head_stride;
  const T* vc = (const T*)a.v + hk * a.head_stride;

  typename M::Q qf;
  M::load_q(qf, (const T*)a.q + b * a.q_stride + (int64_t)(h0 + (col < heads ? col : 0)) * a.D, q,
            a.D, col < heads);
  float m = -INFINITY, l = 0.0f;
  f4 o[M::H][M::VE];
#pragma unroll
  for (int h = 0; h < M::H; ++h)
#pragma unroll
    for (int i = 0; i < M::VE; ++i) o[h][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};

  // chunks split, split + n_splits, ... of the sequence's keys
  for (int64_t c0 = (int64_t)split * a.chunk; c0 < count; c0 += (int64_t)a.n_splits * a.chunk) {
    const int c1 = c0 + a.chunk < count ? (int)c0 + a.chunk : count;
    for (int s0 = (int)c0; s0 < c1; s0 += kKeysAhead) {
      const int n = c1 - s0 < kKeysAhead ? c1 - s0 : kKeysAhead;
      const int nt = (n + M::TK - 1) / M::TK;
      __syncthreads();  // the offsets before these have been used
      for (int i = tid; i < nt * M::TK; i += kAttnThreads) {
        int64_t at = -1;
        if (i < n) {
          const uint32_t key = (uint32_t)(first + s0 + i), c = a.page.div(key);
          const int page = a.table[(int64_t)b * a.max_pages + c];
          if ((uint32_t)page < (uint32_t)a.n_pages)
            at = page * a.page_stride + (int64_t)(key - c * a.page.d) * a.token_stride;
        }
        off[i] = at;
      }
      __syncthreads();
      typename M::K kf;
      if (wave < nt) M::load_k(kf, kc, off + wave * M::TK, lane, a.D);
      for (int t = wave; t < nt; t += kAttnWaves) {
        int64_t at[M::NV];
#pragma unroll
        for (int j = 0; j < M::NV; ++j) at[j] = off[t * M::TK + M::key_of(j, q)];
        typename M::V vf;
        M::load_v(vf, vc, at, lane, a.D);
        float s[M::NV];
        M::scores(s, kf, qf);
        if (t + kAttnWaves < nt) M::load_k(kf, kc, off + (t + kAttnWaves) * M::TK, lane, a.D);
        bool hole = false;
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < M::NV; ++j) {
          s[j] = at[j] < 0 ? -INFINITY : s[j] * a.scale_log2;
          hole |= at[j] < 0;
          mx = fmaxf(mx, s[j]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx);
        const float ref = m_new == -INFINITY ? 0.0f : m_new;  // nothing but masked keys so far
        const float alpha = fast_exp2(m - ref);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < M::NV; ++j) {
          s[j] = fast_exp2(s[j] - ref);
          l += s[j];
        }
        if (__any(alpha != 1.0f)) {
#pragma unroll
          for (int h = 0; h < M::H; ++h)
#pragma unroll
            for (int i = 0; i < M::VE; ++i) o[h][i] *= alpha;
        }
        if (__any(hole)) M::clear_v(vf, at);  // 0 times what a masked row holds is not 0
        M::values(o, s, vf);
      }
    }
  }

  // join the waves: every head's m, l and O
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (q == 0) {
    sm[wave][col] = m;
    sl[wave][col] = l;
  }
#pragma unroll
  for (int h = 0; h < M::H; ++h)
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int i = 0; i < M::VE; i += 4)
        *(f4*)&so[wave][col][16 * M::VE * h + M::VE * (4 * q + r) + i] =
            f4{o[h][i][r], o[h][i + 1][r], o[h][i + 2][r], o[h][i + 3][r]};
  __syncthreads();
  const int per = a.D / 4;
  for (int i = tid; i < heads * per; i += kAttnThreads) {
    const int g = i / per, d = (i - g * per) * 4;
    float mm = -INFINITY;
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) mm = fmaxf(mm, sm[w][g]);
    const float ref = mm == -INFINITY ? 0.0f : mm;
    float ll = 0.0f;
    f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kAttnWaves; ++w) {
      const float f = fast_exp2(sm[w][g] - ref);
      ll = fmaf(f, sl[w][g], ll);
      acc += f * *(const f4*)&so[w][g][d];
    }
    const int64_t row = (int64_t)b * a.Hq + h0 + g;
    if (a.n_splits > 1) {
      *(f4*)(a.part_o + (row * a.n_splits + split) * a.D + d) = acc;
      if (d == 0) {
        a.part_ml[(row * a.n_splits + split) * 2] = mm;
        a.part_ml[(row * a.n_splits + split) * 2 + 1] = ll;
      }
      continue;
    }
    acc *= ll == 0.0f ? 0.0f : 1.0f / ll;
    if constexpr (sizeof(T) == 2)
      *(uint2*)((uint16_t*)a.out + row * a.D + d) =
          make_uint2(f2bf(acc[0]) | (uint32_t)f2bf(acc[1]) << 16,
                     f2bf(acc[2]) | (uint32_t)f2bf(acc[3]) << 16);
    else
      *(f4*)((float*)a.out + row * a.D + d) = acc;
  }
}

// Joins the splits of one query head, four values a thread.
template <typename T>
__global__ __launch_bounds__(64) void attn_join_kernel(AttnArgs a) {
  const int64_t row = (int64_t)blockIdx.y * a.Hq + blockIdx.x;
  const int d = threadIdx.x * 4;
  if (d >= a.D) return;
  int first, count;
  key_range(a, blockIdx.y, first, count);
  const int used = (int)(((int64_t)count + a.chunk - 1) / a.chunk);
  const int n = used < a.n_splits ? used : a.n_splits;
  const float* ml = a.part_ml + row * a.n_splits * 2;
  float mm = -INFINITY;
  for (int i = 0; i < n; ++i) mm = fmaxf(mm, ml[2 * i]);
  const float ref = mm == -INFINITY ? 0.0f : mm;
  float ll = 0.0f;
  f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < n; ++i) {
    const float f = fast_exp2(ml[2 * i] - ref);
    ll = fmaf(f, ml[2 * i + 1], ll);
    acc += f * *(const f4*)(a.part_o + (row * a.n_splits + i) * a.D + d);
  }
  acc *= ll == 0.0f ? 0.0f : 1.0f / ll;
  if constexpr (sizeof(T) == 2)
    *(uint2*)((uint16_t*)a.out + row * a.D + d) =
        make_uint2(f2bf(acc[0]) | (uint32_t)f2bf(acc[1]) << 16,
                   f2bf(acc[2]) | (uint32_t)f2bf(acc[3]) << 16);
  else
    *(f4*)((float*)a.out + row * a.D + d) = acc;
}

int head_tiles(int q_heads, int n_heads) {
  return (q_heads / n_heads + kHeadTile - 1) / kHeadTile;
}

// Most splits that a call with lengths up to max_len makes: enough workgroups
// to fill the chip, but kSplitUnit keys each at least.  Grows with max_len.
int most_splits(int B, int q_heads, int n_heads, int max_len) {
  const int64_t units = (int64_t)B * n_heads * head_tiles(q_heads, n_heads);
  const int64_t want = units == 0 ? 1 : (kSplitGroups + units - 1) / units;
  const int64_t fit = ((int64_t)max_len + kSplitUnit - 1) / kSplitUnit;
  const int64_t n = want < fit ? want : fit;
  return n < 1 ? 1 : (int)n;
}

template <typename T, int DP, bool PAD>
void run_attn(const AttnArgs& a, dim3 grid, hipStream_t s) {
  attn_decode_kernel<T, DP, PAD><<<grid, kAttnThreads, 0, s>>>(a);
}

template <typename T>
hipError_t run_attn_t(const AttnArgs& a, int B, hipStream_t s) {
  const dim3 grid(a.n_splits * a.H * a.tiles, B);
  if (a.D == 64) run_attn<T, 64, false>(a, grid, s);
  else if (a.D < 64) run_attn<T, 64, true>(a, grid, s);
  else if (a.D == 128) run_attn<T, 128, false>(a, grid, s);
  else if (a.D < 128) run_attn<T, 128, true>(a, grid, s);
  else if (a.D == 256) run_attn<T, 256, false>(a, grid, s);
  else run_attn<T, 256, true>(a, grid, s);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || a.n_splits == 1) return err;
  attn_join_kernel<T><<<dim3(a.Hq, B), 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t attn_decode_workspace(int B, int q_heads, int n_heads, int dim, int max_len) {
  const int n = most_splits(B, q_heads, n_heads, max_len);
  return n == 1 ? 0 : (size_t)B * q_heads * n * (dim + 2) * sizeof(float);
}

hipError_t launch_attn_decode(const void* q, int64_t q_stride, int B, int q_heads,
                              const d2moe_kv_cache* c, const int32_t* table, int max_pages,
                              const int32_t* lengths, int max_len, int window, float scale,
                              void* out, void* ws, hipStream_t s) {
  if (B == 0) return hipSuccess;
  AttnArgs a{};
  a.q = q, a.k = c->k, a.v = c->v, a.q_stride = q_stride, a.page_stride = c->page_stride;
  a.token_stride = c->token_stride, a.head_stride = c->head_stride;
  a.table = table, a.lengths = lengths, a.page = fast_div(c->page_size);
  a.n_pages = c->n_pages, a.max_pages = max_pages, a.Hq = q_heads, a.H = c->n_heads;
  a.G = q_heads / c->n_heads, a.tiles = head_tiles(q_heads, c->n_heads), a.D = c->head_dim;
  a.window = window;
  const int keys = window > 0 && window < max_len ? window : max_len;
  const int n = most_splits(B, q_heads, c->n_heads, keys);
  const int units = (int)(((int64_t)keys + n - 1) / n + kSplitUnit - 1) / kSplitUnit;
  a.chunk = (units < 1 ? 1 : units) * kSplitUnit;
  a.n_splits = keys > 0 ? (int)(((int64_t)keys + a.chunk - 1) / a.chunk) : 1;
  a.scale_log2 = scale * 1.44269504088896340736f;
  a.out = out;
  a.part_o = (float*)ws;
  a.part_ml = (float*)ws + (size_t)B * q_heads * a.n_splits * a.D;
  return c->dtype == D2MOE_BF16 ? run_attn_t<uint16_t>(a, B, s) : run_attn_t<float>(a, B, s);
}

}  // namespace d2moe
