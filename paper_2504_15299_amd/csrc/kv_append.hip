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
template <bool PAST, typename T>
__device__ inline void put(T* p, const T& v) {
  if constexpr (PAST) {
    // 32-byte packs are stored in two
    constexpr int kWords = sizeof(T) < 16 ? sizeof(T) / 4 : 4;
    typedef uint32_t words __attribute__((ext_vector_type(kWords)));
    struct Parts {
      words w[sizeof(T) / 4 / kWords];
    };
    const Parts x = __builtin_bit_cast(Parts, v);
#pragma unroll
    for (int i = 0; i < (int)(sizeof(T) / 4 / kWords); ++i)
      __builtin_nontemporal_store(x.w[i], (words*)p + i);
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
// places that it read.
struct NormArgs {
  AppendArgs a;
  const float *qw, *kw;  // [D] or null
  int R;
  float eps;
  bool interleaved;
};

__device__ inline void turn(float& a, float& b, float cos, float sin) {
  const float x = a * cos - b * sin;
  b = b * cos + a * sin;
  a = x;
}

template <typename TI, typename TO, int N, int LANES, bool PAST>
__global__ __launch_bounds__(kAppendThreads) void kv_append_norm_kernel(NormArgs g) {
  const AppendArgs& a = g.a;
  const int item = blockIdx.x * kAppendThreads + threadIdx.x;
  const int head = item / LANES, l = item & (LANES - 1);
  if (head >= a.Hq + 2 * a.H) return;
  const int pairs = g.R / 2;           // of a head
  const bool live = 2 * N * l < a.D;   // (LANES is a power of two)
  const bool turns = N * l < pairs;
  const int first = !live ? 0 : turns && !g.interleaved ? N * l : 2 * N * l;
  const int second = turns && !g.interleaved ? first + pairs : first + N;
  const bool key = head >= a.Hq && head < a.Hq + a.H;
  const float* weight = head < a.Hq ? g.qw : key ? g.kw : nullptr;
  Pack<float, N> wu, ww;
  if (weight) {
    wu = *(const Pack<float, N>*)(weight + first);
    ww = *(const Pack<float, N>*)(weight + second);
  }
  for (int t = blockIdx.y; t < a.N; t += gridDim.y) {
    const int pos = a.positions[t];
    const bool in = pos >= 0 && pos < a.n_rot;
    const TI* src;
    TO* dst;
    if (head < a.Hq) {
      src = (const TI*)a.q + t * a.q_stride + (int64_t)head * a.D;
      dst = (TO*)a.q_out + ((int64_t)t * a.Hq + head) * a.D;
    } else {
      const int h = head - a.Hq - (key ? 0 : a.H);
      const int seq = a.token_seq ? a.token_seq[t] : t;
      if (pos < 0 || (a.cos && !in) || seq < 0 || seq >= a.n_seqs) continue;
      const uint32_t col = a.page.div((uint32_t)pos);
      if (col >= (uint32_t)a.max_pages) continue;
      const int page = a.table[(int64_t)seq * a.max_pages + col];
      if ((uint32_t)page >= (uint32_t)a.n_pages) continue;
      const int64_t at = page * a.page_stride +
                         (int64_t)((uint32_t)pos - col * a.page.d) * a.token_stride +
                         h * a.head_stride;
      src = (const TI*)(key ? a.k : a.v) + t * a.kv_stride + (int64_t)h * a.D;
      dst = (TO*)(key ? a.kc : a.vc) + at;
    }
    const Pack<TI, N> x = *(const Pack<TI, N>*)(src + first);
    const Pack<TI, N> y = *(const Pack<TI, N>*)(src + second);
    float u[N], v[N], sum = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      u[e] = to_f(x.v[e]);
      v[e] = to_f(y.v[e]);
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
    if (turns && in && (key || head < a.Hq)) {
      const Pack<float, N> c = *(const Pack<float, N>*)(a.cos + (int64_t)pos * pairs + N * l);
      const Pack<float, N> s = *(const Pack<float, N>*)(a.sin + (int64_t)pos * pairs + N * l);
      if (g.interleaved) {
#pragma unroll
        for (int e = 0; e < N / 2; ++e) {
          turn(u[2 * e], u[2 * e + 1], c.v[e], s.v[e]);
          turn(v[2 * e], v[2 * e + 1], c.v[N / 2 + e], s.v[N / 2 + e]);
        }
      } else {
#pragma unroll
        for (int e = 0; e < N; ++e) turn(u[e], v[e], c.v[e], s.v[e]);
      }
    }
    if (!live) continue;
    Pack<TO, N> o, w;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      from_f(u[e], o.v[e]);
      from_f(v[e], w.v[e]);
    }
    put<PAST>((Pack<TO, N>*)(dst + first), o);
    put<PAST>((Pack<TO, N>*)(dst + second), w);
  }
}

template <typename TI, typename TO, int N, int LANES>
hipError_t run_norm_l(const NormArgs& g, hipStream_t s) {
  const int items = (g.a.Hq + 2 * g.a.H) * LANES;
  const dim3 grid((items + kAppendThreads - 1) / kAppendThreads, g.a.N < 65535 ? g.a.N : 65535);
  if (g.a.N <= 256)
    kv_append_norm_kernel<TI, TO, N, LANES, false><<<grid, kAppendThreads, 0, s>>>(g);
  else
    kv_append_norm_kernel<TI, TO, N, LANES, true><<<grid, kAppendThreads, 0, s>>>(g);
  return hipGetLastError();
}

template <typename TI, typename TO, int N>
hipError_t run_norm_n(const NormArgs& g, hipStream_t s) {
  const int lanes = g.a.D / (2 * N);
  if (lanes <= 64 / N) return run_norm_l<TI, TO, N, 64 / N>(g, s);    // D <= 128
  return run_norm_l<TI, TO, N, 128 / N>(g, s);
}

// Packs of 8, 4 or 2 values, as the rotated part and the rest both divide into
// pairs of them (D % 8 == 0, R % 4 == 0).
template <typename TI, typename TO>
hipError_t run_norm(const NormArgs& g, hipStream_t s) {
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
  const NormArgs g{append_args(q, q_stride, q_heads, k, v, kv_stride, N, c, table, n_seqs, max_pages,
                               positions, token_seq, cos, sin, cos ? n_rot : 0, q_out),
                   q_weight, k_weight, cos ? rot_dim : 0, eps, interleaved};
  const bool xb = xd == D2MOE_BF16, cb = c->dtype == D2MOE_BF16;
  if (xb) return cb ? run_norm<uint16_t, uint16_t>(g, s) : run_norm<uint16_t, float>(g, s);
  return cb ? run_norm<float, uint16_t>(g, s) : run_norm<float, float>(g, s);
}

}  // namespace d2moe
