// New tokens into the paged key-value cache, with the rotary rotation of
// their queries and keys:
//   (a, b) = (x[i], x[i + D/2])  ->  (a cos_i - b sin_i, b cos_i + a sin_i)
// and plain copies of the value rows; in a second form with the RMS norms of the
// query and key heads before it, and a rotation of part of a head or of
// neighbouring values.  Memory-bound: every row is read and written once.
#include "decoder.h"

namespace d2moe {
namespace {

constexpr int kAppendThreads = 256;

template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
  T v[N];
};

__device__ inline float to_f(uint16_t b) { return bf2f(b); }
__device__ inline float to_f(float f) { return f; }
__device__ inline void from_f(float f, uint16_t& o) { o = f2bf(f); }
__device__ inline void from_f(float f, float& o) { o = f; }

struct AppendArgs {
  const void *q, *k, *v;
  int64_t q_stride, kv_stride, page_stride, token_stride, head_stride;
  void *kc, *vc, *q_out;
  const int32_t *table, *positions, *token_seq;
  const float *cos, *sin;
  FastDiv page;
  int N, Hq, H, D, n_pages, n_seqs, max_pages, n_rot;
};

// One thread takes N values of the first half of a head and the N that go
// with them in the second.  Workgroups walk a token's heads along x (queries,
// keys, values), tokens along y.
// PAST: many tokens' rows leave the caches before they are read again and are
// stored past them (1024 tokens, 32 and 8 heads of 128, bf16: 7.9 -> 6.6 us; 8192:
// 41.8 -> 41.0 us, 4.9 TB/s).
template <typename T>
struct Words {  // of 16 bytes at most
  static constexpr int kEach = sizeof(T) < 16 ? sizeof(T) / 4 : 4, kN = sizeof(T) / 4 / kEach;
  typedef uint32_t words __attribute__((ext_vector_type(kEach)));
  words w[kN];
};

template <bool PAST, typename T>
__device__ inline void put(T* p, const T& v) {
  if constexpr (PAST) {
    typedef Words<T> W;
    const W x = __builtin_bit_cast(W, v);
#pragma unroll
    for (int i = 0; i < W::kN; ++i)
      __builtin_nontemporal_store(x.w[i], (typename W::words*)p + i);
  } else {
    *p = v;
  }
}

template <typename TI, typename TO, int N, bool PAST>
__global__ __launch_bounds__(kAppendThreads) void kv_append_kernel(AppendArgs a) {
  const int half = a.D / 2, per = half / N;
  const int item = blockIdx.x * kAppendThreads + threadIdx.x;
  const int head = item / per, i = (item - head * per) * N;
  if (head >= a.Hq + 2 * a.H) return;
  for (int t = blockIdx.y; t < a.N; t += gridDim.y) {
    const int pos = a.positions[t];
    const TI* src;
    TO* dst;
    bool rotate = a.cos != nullptr;
    if (rotate && (pos < 0 || pos >= a.n_rot)) {
      if (head >= a.Hq) continue;  // not written
      rotate = false;
    }
    if (head < a.Hq) {
      src = (const TI*)a.q + t * a.q_stride + (int64_t)head * a.D;
      dst = (TO*)a.q_out + ((int64_t)t * a.Hq + head) * a.D;
    } else {
      const bool key = head < a.Hq + a.H;
      const int h = head - a.Hq - (key ? 0 : a.H);
      const int seq = a.token_seq ? a.token_seq[t] : t;
      if (pos < 0 || seq < 0 || seq >= a.n_seqs) continue;
      const uint32_t col = a.page.div((uint32_t)pos);
      if (col >= (uint32_t)a.max_pages) continue;
      const int page = a.table[(int64_t)seq * a.max_pages + col];
      if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
      const int64_t at = page * a.page_stride +
                         (int64_t)((uint32_t)pos - col * a.page.d) * a.token_stride +
                         h * a.head_stride;
      src = (const TI*)(key ? a.k : a.v) + t * a.kv_stride + (int64_t)h * a.D;
      dst = (TO*)(key ? a.kc : a.vc) + at;
      rotate = rotate && key;
    }
    const Pack<TI, N> x = *(const Pack<TI, N>*)(src + i), y = *(const Pack<TI, N>*)(src + half + i);
    Pack<TO, N> u, w;
    if (rotate) {
      const Pack<float, N> c = *(const Pack<float, N>*)(a.cos + (int64_t)pos * half + i);
      const Pack<float, N> s = *(const Pack<float, N>*)(a.sin + (int64_t)pos * half + i);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float p = to_f(x.v[e]), r = to_f(y.v[e]);
        from_f(p * c.v[e] - r * s.v[e], u.v[e]);
        from_f(r * c.v[e] + p * s.v[e], w.v[e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        from_f(to_f(x.v[e]), u.v[e]);
        from_f(to_f(y.v[e]), w.v[e]);
      }
    }
    put<PAST>((Pack<TO, N>*)(dst + i), u);
    put<PAST>((Pack<TO, N>*)(dst + half + i), w);
  }
}

template <typename TI, typename TO, int N>
hipError_t run_append_n(const AppendArgs& a, hipStream_t s) {
  const int items = (a.Hq + 2 * a.H) * (a.D / 2 / N);
  const dim3 grid((items + kAppendThreads - 1) / kAppendThreads, a.N < 65535 ? a.N : 65535);
  if (a.N <= 256)
    kv_append_kernel<TI, TO, N, false><<<grid, kAppendThreads, 0, s>>>(a);
  else
    kv_append_kernel<TI, TO, N, true><<<grid, kAppendThreads, 0, s>>>(a);
  return hipGetLastError();
}

template <typename TI, typename TO>
hipError_t run_append(const AppendArgs& a, hipStream_t s) {
  // 16-byte accesses of bf16 need halves of 8 values; 4 always fit (D % 8 == 0)
  if constexpr (sizeof(TI) == 2 || sizeof(TO) == 2)
    if (a.D % 16 == 0) return run_append_n<TI, TO, 8>(a, s);
  return run_append_n<TI, TO, 4>(a, s);
}

// The form with norms: of a query or key head x
//   n = w x / sqrt(mean_i x_i^2 + eps),
// then pairs among its first R values rotated, (i, i + R/2) or (2 i, 2 i + 1), the
// others as they are.  A head belongs to LANES neighbouring lanes of one wave, each
// with 2 N of its values: first the pairs, N a lane, then what is not rotated.  The
// sum of squares crosses the lanes; nothing else does, and each lane writes the
// places that it read.  A wave takes 64 / LANES heads of one token, neighbours in
// memory, at a time, and keeps these heads and their weights from token to token.
// Memory-bound: 8192 tokens of 32 and 8 heads of 128, bf16, take 42.5 us, 4.7 TB/s (a
// scaled copy of as many bytes 37.5); 16 tokens 3.5 us, which is latency.  The heads'
// loads are under way before the token's position is waited for (one after the other:
// 52 us), rows are stored past the caches (through them 48 us and more; 16 tokens and the
// attention that reads them next 20.1 us, through them 19.9, 256 tokens 189 for 192), and
// the 5 workgroups a compute unit that the registers leave room for go over the tokens (6:
// 48.5 us, 7: 45.4, one for each 4 waves' work 47).  Two of a wave's heads in flight at once
// gain nothing (46 us).
struct NormArgs {
  AppendArgs a;
  const float *qw, *kw;  // [D] or null
  FastDiv by_turns;  // by the waves that a token takes
  int R, step;
  float eps;
  bool interleaved;
};

constexpr int kNormGroups = 5, kMostGroups = 256 * kNormGroups;  // a compute unit, all

__device__ inline void turn_pair(float& a, float& b, float cos, float sin) {
  const float x = a * cos - b * sin;
  b = b * cos + a * sin;
  a = x;
}

template <typename TI, typename TO, int N, int LANES>
__global__ __launch_bounds__(kAppendThreads, kNormGroups) void kv_append_norm_kernel(NormArgs g) {
  typedef Words<Pack<TI, N>> W;
  constexpr int kHeads = 64 / LANES;  // side by side in a wave
  constexpr int kWaves = kAppendThreads / 64;
  const AppendArgs& a = g.a;
  const int lane = threadIdx.x & 63, l = lane & (LANES - 1);
  const int pairs = g.R / 2;          // of a head
  const bool live = 2 * N * l < a.D;  // (LANES is a power of two)
  const bool turns = N * l < pairs;
  const int first = !live ? 0 : turns && !g.interleaved ? N * l : 2 * N * l;
  const int second = turns && !g.interleaved ? first + pairs : first + N;
  const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * kWaves + threadIdx.x / 64);
  const uint32_t from = g.by_turns.div(wave), turn = wave - from * g.by_turns.d;
  const int mine = (int)turn * kHeads + lane / LANES, last = a.Hq + 2 * a.H - 1;
  const int head = mine < last ? mine : last, h = head - a.Hq;
  const bool query = h < 0, key = !query && h < a.H;
  const float* weight = query ? g.qw : key ? g.kw : nullptr;
  Pack<float, N> wu, ww;
  if (weight) {
    wu = *(const Pack<float, N>*)(weight + first);
    ww = *(const Pack<float, N>*)(weight + second);
  }
  const TI* src = (const TI*)a.q + (int64_t)head * a.D;
  if (!query) src = (const TI*)(key ? a.k : a.v) + (int64_t)(key ? h : h - a.H) * a.D;
  const int64_t stride = query ? a.q_stride : a.kv_stride;
  for (uint32_t t = from; t < (uint32_t)a.N; t += g.step) {
    const int pos = a.positions[t], given = (a.token_seq ? a.token_seq : a.positions)[t];
    const int seq = a.token_seq ? given : (int)t;
    // (as words: what is unpacked here would be waited for here)
    const W x = *(const W*)(src + (int64_t)t * stride + first);
    const W y = *(const W*)(src + (int64_t)t * stride + second);
    const bool in = pos >= 0 && pos < a.n_rot;
    Pack<float, N> c, s;
    if (turns && in) {
      c = *(const Pack<float, N>*)(a.cos + (int64_t)pos * pairs + N * l);
      s = *(const Pack<float, N>*)(a.sin + (int64_t)pos * pairs + N * l);
    }
    int64_t at = -1;  // the token's place in a head of the cache
    if (pos >= 0 && (!a.cos || in) && seq >= 0 && seq < a.n_seqs) {
      const uint32_t col = a.page.div((uint32_t)pos);
      if (col < (uint32_t)a.max_pages) {
        const int page = a.table[(int64_t)seq * a.max_pages + col];
        if ((uint32_t)page < (uint32_t)a.n_pages)
          at = page * a.page_stride + (int64_t)((uint32_t)pos - col * a.page.d) * a.token_stride;
      }
    }
    const Pack<TI, N> xv = __builtin_bit_cast(Pack<TI, N>, x);
    const Pack<TI, N> yv = __builtin_bit_cast(Pack<TI, N>, y);
    float u[N], v[N], sum = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      u[e] = to_f(xv.v[e]);
      v[e] = to_f(yv.v[e]);
      sum = fmaf(u[e], u[e], fmaf(v[e], v[e], sum));
    }
    if (!live) sum = 0.0f;
#pragma unroll
    for (int off = 1; off < LANES; off *= 2) sum += __shfl_xor(sum, off, 64);
    if (weight) {
      const float r = 1.0f / sqrtf(sum / (float)a.D + g.eps);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        u[e] *= r * wu.v[e];
        v[e] *= r * ww.v[e];
      }
    }
    if (turns && in && (query || key)) {
      if (g.interleaved) {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          turn_pair(u[2 * e], u[2 * e + 1], c.v[e], s.v[e]);
          turn_pair(v[2 * e], v[2 * e + 1], c.v[N / 2 + e], s.v[N / 2 + e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) turn_pair(u[e], v[e], c.v[e], s.v[e]);
      }
    }
    if (!live || mine > last || (!query && at < 0)) continue;
    TO* dst = (TO*)a.q_out + ((int64_t)t * a.Hq + head) * a.D;
    if (!query) dst = (TO*)(key ? a.kc : a.vc) + at + (key ? h : h - a.H) * a.head_stride;
    Pack<TO, N> o, w;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      from_f(u[e], o.v[e]);
      from_f(v[e], w.v[e]);
    }
    put<true>((Pack<TO, N>*)(dst + first), o);
    put<true>((Pack<TO, N>*)(dst + second), w);
  }
}

template <typename TI, typename TO, int N, int LANES>
hipError_t run_norm_l(NormArgs& g, hipStream_t s) {
  constexpr int kHeads = 64 / LANES, kWaves = kAppendThreads / 64;
  const int turns = (g.a.Hq + 2 * g.a.H + kHeads - 1) / kHeads;
  int64_t groups = ((int64_t)g.a.N * turns + kWaves - 1) / kWaves;
  g.by_turns = fast_div(turns), g.step = g.a.N;
  if (groups > kMostGroups) {  // a wave keeps its heads
    groups = turns < kMostGroups ? kMostGroups / turns * turns : turns;
    g.step = (int)(groups * kWaves / turns);
  }
  kv_append_norm_kernel<TI, TO, N, LANES><<<(int)groups, kAppendThreads, 0, s>>>(g);
  return hipGetLastError();
}

template <typename TI, typename TO, int N>
hipError_t run_norm_n(NormArgs& g, hipStream_t s) {
  const int lanes = g.a.D / (2 * N);
  if (lanes <= 32 / N) return run_norm_l<TI, TO, N, 32 / N>(g, s);  // D <= 64
  if (lanes <= 64 / N) return run_norm_l<TI, TO, N, 64 / N>(g, s);  // D <= 128
  return run_norm_l<TI, TO, N, 128 / N>(g, s);
}

// Packs of 8, 4 or 2 values, as the rotated part and the rest both divide into
// pairs of them (D % 8 == 0, R % 4 == 0).
template <typename TI, typename TO>
hipError_t run_norm(NormArgs& g, hipStream_t s) {
  if (g.a.D % 16 == 0 && g.R % 16 == 0) return run_norm_n<TI, TO, 8>(g, s);
  if (g.R % 8 == 0) return run_norm_n<TI, TO, 4>(g, s);
  return run_norm_n<TI, TO, 2>(g, s);
}

AppendArgs append_args(const void* q, int64_t q_stride, int q_heads, const void* k, const void* v,
                       int64_t kv_stride, int N, const d2moe_kv_cache* c, const int32_t* table,
                       int n_seqs, int max_pages, const int32_t* positions,
                       const int32_t* token_seq, const float* cos, const float* sin, int n_rot,
                       void* q_out) {
  AppendArgs a{};
  a.q = q, a.k = k, a.v = v, a.q_stride = q_stride, a.kv_stride = kv_stride;
  a.page_stride = c->page_stride, a.token_stride = c->token_stride;
  a.head_stride = c->head_stride;
  a.kc = c->k, a.vc = c->v, a.q_out = q_out;
  a.table = table, a.positions = positions, a.token_seq = token_seq, a.cos = cos, a.sin = sin;
  a.page = fast_div(c->page_size);
  a.N = N, a.Hq = q ? q_heads : 0, a.H = c->n_heads, a.D = c->head_dim, a.n_pages = c->n_pages;
  a.n_seqs = n_seqs, a.max_pages = max_pages, a.n_rot = n_rot;
  return a;
}

}  // namespace

hipError_t launch_kv_append(const void* q, int64_t q_stride, int q_heads, const void* k,
                            const void* v, int64_t kv_stride, d2moe_dtype xd, int N,
                            const d2moe_kv_cache* c, const int32_t* table, int n_seqs,
                            int max_pages, const int32_t* positions, const int32_t* token_seq,
                            const float* cos, const float* sin, int n_rot, void* q_out,
                            hipStream_t s) {
  if (N == 0) return hipSuccess;
  const AppendArgs a = append_args(q, q_stride, q_heads, k, v, kv_stride, N, c, table, n_seqs,
                                   max_pages, positions, token_seq, cos, sin, n_rot, q_out);
  const bool xb = xd == D2MOE_BF16, cb = c->dtype == D2MOE_BF16;
  if (xb) return cb ? run_append<uint16_t, uint16_t>(a, s) : run_append<uint16_t, float>(a, s);
  return cb ? run_append<float, uint16_t>(a, s) : run_append<float, float>(a, s);
}

hipError_t launch_kv_append_norm(const void* q, int64_t q_stride, int q_heads, const void* k,
                                 const void* v, int64_t kv_stride, d2moe_dtype xd, int N,
                                 const d2moe_kv_cache* c, const int32_t* table, int n_seqs,
                                 int max_pages, const int32_t* positions, const int32_t* token_seq,
                                 const float* q_weight, const float* k_weight, float eps,
                                 const float* cos, const float* sin, int n_rot, int rot_dim,
                                 bool interleaved, void* q_out, hipStream_t s) {
  if (N == 0) return hipSuccess;
  NormArgs g{append_args(q, q_stride, q_heads, k, v, kv_stride, N, c, table, n_seqs, max_pages,
                               positions, token_seq, cos, sin, cos ? n_rot : 0, q_out),
                   q_weight, k_weight, FastDiv{}, cos ? rot_dim : 0, 0, eps, interleaved};
  const bool xb = xd == D2MOE_BF16, cb = c->dtype == D2MOE_BF16;
  if (xb) return cb ? run_norm<uint16_t, uint16_t>(g, s) : run_norm<uint16_t, float>(g, s);
  return cb ? run_norm<float, uint16_t>(g, s) : run_norm<float, float>(g, s);
}

}  // namespace d2moe
