// New tokens into the paged key-value cache, with the rotary rotation of
// their queries and keys:
//   (a, b) = (x[i], x[i + D/2])  ->  (a cos_i - b sin_i, b cos_i + a sin_i)
// and plain copies of the value rows.  Memory-bound: every row is read and
// written once.
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

}  // namespace

hipError_t launch_kv_append(const void* q, int64_t q_stride, int q_heads, const void* k,
                            const void* v, int64_t kv_stride, d2moe_dtype xd, int N,
                            const d2moe_kv_cache* c, const int32_t* table, int n_seqs,
                            int max_pages, const int32_t* positions, const int32_t* token_seq,
                            const float* cos, const float* sin, int n_rot, void* q_out,
                            hipStream_t s) {
  if (N == 0) return hipSuccess;
  AppendArgs a{};
  a.q = q, a.k = k, a.v = v, a.q_stride = q_stride, a.kv_stride = kv_stride;
  a.page_stride = c->page_stride, a.token_stride = c->token_stride;
  a.head_stride = c->head_stride;
  a.kc = c->k, a.vc = c->v, a.q_out = q_out;
  a.table = table, a.positions = positions, a.token_seq = token_seq, a.cos = cos, a.sin = sin;
  a.page = fast_div(c->page_size);
  a.N = N, a.Hq = q ? q_heads : 0, a.H = c->n_heads, a.D = c->head_dim, a.n_pages = c->n_pages;
  a.n_seqs = n_seqs, a.max_pages = max_pages, a.n_rot = n_rot;
  const bool xb = xd == D2MOE_BF16, cb = c->dtype == D2MOE_BF16;
  if (xb) return cb ? run_append<uint16_t, uint16_t>(a, s) : run_append<uint16_t, float>(a, s);
  return cb ? run_append<float, uint16_t>(a, s) : run_append<float, float>(a, s);
}

}  // namespace d2moe
