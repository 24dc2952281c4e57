// One token per row of logits, by temperature, top-k, top-p, min-p and a given random
// number.  With w_i = exp((l_i - max l) / t) and the tokens in descending order of l
// (ties: ascending index), every bound keeps a beginning of that order, so the kept
// tokens are one, of weight W = the least of the bounds' sums; the token is the first
// whose running sum passes u W.  All of it is one question, asked up to three times:
// the first token whose running count or sum reaches a target.
//
// Nothing is sorted.  A histogram over log2 w (counts and weights) says in which of
// 2048 bins the target lies, and only that bin's tokens, some hundred, are ranked
// against each other.  A bin with more than fit the list is divided by its keys until
// they fit or are all equal.
//
// Weights are integers, w in units of 2^-frac, as small as V of them leave room for
// in 64 bits (2^-47 at 32000 tokens).  Their sums are exact, so that no order of
// additions turns a choice; a token below half a unit is never drawn.
#include "decoder.h"

namespace d2moe {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048, kList = 1024;

struct SampleArgs {
  const void* logits;
  int64_t stride;
  int V, frac;
  const float *u, *temperature;
  const int32_t* top_k;
  const float *top_p, *min_p;
  int32_t* tokens;
  float* probs;
};

// Order of binary32 values as unsigned numbers, NaN and -infinity (never drawn) 0.
__device__ inline uint32_t key_of(float l) {
  if (!(l > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(l + 0.0f);  // (-0 is 0)
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ inline float value_of(uint32_t key) {
  return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key);
}

// Values l with their indexes, all of a row once, by kThreads threads: a thread takes
// whole 16 bytes where the row's memory has them.
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return bf2f(*p); }
template <typename T>
struct RowOf {
  static constexpr int PER = 16 / sizeof(T);
  const T* p;
  int V, skip, chunks;  // elements of the first 16 bytes that lie before the row
  __device__ RowOf(const T* row, int V) : p(row), V(V) {
    skip = (int)(((uintptr_t)row & 15) / sizeof(T));
    chunks = (V + skip + PER - 1) / PER;
  }
  __device__ void load(int c, float (&l)[PER], int& i0) const {  // outside: -infinity
    i0 = c * PER - skip;
    if (i0 >= 0 && i0 + PER <= V) {
      const uint4 x = *(const uint4*)(p + i0);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int e = 0; e < PER; ++e)
        l[e] = sizeof(T) == 4 ? __uint_as_float(w[e / (PER / 4)])
                              : __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        l[e] = i0 + e >= 0 && i0 + e < V ? load1(p + i0 + e) : -INFINITY;
    }
  }
  template <typename F>
  __device__ void each(F f) const {
    for (int c = threadIdx.x; c < chunks; c += kThreads) {
      float l[PER];
      int i0;
      load(c, l, i0);
#pragma unroll
      for (int e = 0; e < PER; ++e) f(l[e], i0 + e);
    }
  }
};

// 2^y for -64 < y <= 0 from a table of 2^(i / 64) and the series of 2^r, |r| <= 1/128,
// to the fifth power (the next term is 2^-55 of the whole).
__device__ inline double exp2_of(double y, const double* table) {
  constexpr double kShift = 6755399441055744.0;  // 1.5 2^52: whole numbers in the last bits
  const double at = fma(y, 64.0, kShift);
  const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, at);
  const double r = fma(at - kShift, -1.0 / 64, y);
  double s = 0.0013333558146428441;  // (ln 2)^5 / 5!, and so on
  s = fma(s, r, 0.009618129107628477);
  s = fma(s, r, 0.055504108664821576);
  s = fma(s, r, 0.2402265069591007);
  s = fma(s, r, 0.6931471805599453);
  s = fma(s, r, 1.0) * table[n & 63];
  return __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, s) +
                                        ((uint64_t)(int64_t)(n >> 6) << 52));
}

struct Weights {
  const double* table;
  float top;
  double per;  // 1 / (t ln 2)
  int frac;
  double bins;  // per unit of log2
  // log2 w, NaN where the weight is 0 whatever the value
  __device__ double log2w(float l) const {
    return l == top ? 0.0 : ((double)l - (double)top) * per;
  }
  __device__ bool counts(double y) const { return y > -(double)(frac + 1); }
  __device__ double weight(double y) const { return exp2_of(y, table); }
  __device__ uint64_t units(double w) const {  // rounded to nearest
    const double x = __builtin_bit_cast(double, __builtin_bit_cast(uint64_t, w) +
                                                    ((uint64_t)frac << 52));
    return __builtin_bit_cast(uint64_t, x + 4503599627370496.0) & 0xfffffffffffffull;
  }
  __device__ int bin(double y) const {
    const int b = (int)(-y * bins);
    return b < kBins ? b : kBins - 1;
  }
};

typedef unsigned long long u64;

struct Lds {
  double table[64];
  u64 weight[2][kBins];  // inclusive sums after scan(); [1]: of a bin's parts
  int count[2][kBins];
  u64 order[kList], units[kList];  // ~key and index; the weight
  u64 wave_w[kWaves];
  int wave_n[kWaves];
  int n;
  uint32_t lo, hi;
  // what select() found
  int bin, in_bin;
  u64 base_n, base_w;
  u64 found, found_w;
};

__device__ inline u64 shfl_up64(u64 v, int d) {
  const uint32_t lo = __shfl_up((uint32_t)v, d, 64), hi = __shfl_up((uint32_t)(v >> 32), d, 64);
  return (u64)hi << 32 | lo;
}
__device__ inline u64 shfl_xor64(u64 v, int d) {
  const uint32_t lo = __shfl_xor((uint32_t)v, d, 64), hi = __shfl_xor((uint32_t)(v >> 32), d, 64);
  return (u64)hi << 32 | lo;
}

// count[h] and weight[h] to inclusive sums.
__device__ void scan(Lds& s, int h) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n0 = s.count[h][2 * tid], n1 = n0 + s.count[h][2 * tid + 1];
  const u64 w0 = s.weight[h][2 * tid], w1 = w0 + s.weight[h][2 * tid + 1];
  int n = n1;
  u64 w = w1;
  for (int d = 1; d < 64; d *= 2) {
    const int on = __shfl_up(n, d, 64);
    const u64 ow = shfl_up64(w, d);
    if (lane >= d) n += on, w += ow;
  }
  if (lane == 63) s.wave_n[wave] = n, s.wave_w[wave] = w;
  __syncthreads();
  for (int i = 0; i < wave; ++i) n += s.wave_n[i], w += s.wave_w[i];
  s.count[h][2 * tid] = n - n1 + n0;
  s.count[h][2 * tid + 1] = n;
  s.weight[h][2 * tid] = w - w1 + w0;
  s.weight[h][2 * tid + 1] = w;
  __syncthreads();
}

// The bin of histogram h whose running count (by_count) or weight is the first to reach
// target, base_n and base_w the sums before it.
__device__ void locate(Lds& s, int h, bool by_count, u64 target) {
  for (int j = 2 * threadIdx.x; j <= 2 * (int)threadIdx.x + 1; ++j) {
    const u64 n = s.count[h][j], n0 = j ? s.count[h][j - 1] : 0;
    const u64 w = s.weight[h][j], w0 = j ? s.weight[h][j - 1] : 0;
    if (by_count ? n0 < target && target <= n : w0 < target && target <= w) {
      s.bin = j;
      s.in_bin = (int)(n - n0);
      s.base_n = n0;
      s.base_w = w0;
    }
  }
  __syncthreads();
}

// Among the tokens that `in` takes (n of them, at most kList), the first whose running
// count or weight reaches target, base_n and base_w before the first.
template <typename T, typename In>
__device__ void rank(Lds& s, const RowOf<T>& row, const Weights& x, In in, bool by_count,
                     u64 target, u64 base_n, u64 base_w) {
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
  row.each([&](float l, int i) {
    const double y = x.log2w(l);
    if (!x.counts(y)) return;
    const uint32_t key = key_of(l);
    if (!in(y, key)) return;
    const u64 units = x.units(x.weight(y));
    if (units == 0) return;
    const int at = atomicAdd(&s.n, 1);
    s.order[at] = (u64)~key << 32 | (uint32_t)i;
    s.units[at] = units;
  });
  __syncthreads();
  const int n = s.n, part = threadIdx.x & 15;
  for (int i0 = 0; i0 < n; i0 += kThreads / 16) {
    const int i = i0 + (threadIdx.x >> 4);
    const u64 mine = i < n ? s.order[i] : 0;
    u64 count = 0, sum = 0;
    for (int j = part; j < n; j += 16)
      if (s.order[j] <= mine) count += 1, sum += s.units[j];
    for (int d = 1; d < 16; d *= 2) {
      count += shfl_xor64(count, d);
      sum += shfl_xor64(sum, d);
    }
    if (i < n && part == 0) {
      const u64 own = by_count ? 1 : s.units[i], run = by_count ? base_n + count : base_w + sum;
      if (run >= target && run - own < target) {
        s.found = mine;
        s.found_w = base_w + sum;
      }
    }
  }
  __syncthreads();
}

// The j-th token in index order, from 1, of one key.
template <typename T>
__device__ void nth(Lds& s, const RowOf<T>& row, uint32_t key, u64 j) {
  constexpr int PER = RowOf<T>::PER;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 before = 0;
  for (int c0 = 0; c0 < row.chunks && before < j; c0 += kThreads) {
    float l[PER];
    int i0 = 0, mine = 0;
    const bool have = c0 + (int)threadIdx.x < row.chunks;
    if (have) {
      row.load(c0 + threadIdx.x, l, i0);
#pragma unroll
      for (int e = 0; e < PER; ++e) mine += key_of(l[e]) == key;
    }
    int n = mine;
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(n, d, 64);
      if (lane >= d) n += o;
    }
    __syncthreads();
    if (lane == 63) s.wave_n[wave] = n;
    __syncthreads();
    int all = 0;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) n += s.wave_n[w];
      all += s.wave_n[w];
    }
    u64 run = before + n - mine;
    if (have && run < j && j <= run + mine)
#pragma unroll
      for (int e = 0; e < PER; ++e)
        if (key_of(l[e]) == key && ++run == j) s.found = (u64)~key << 32 | (uint32_t)(i0 + e);
    before += all;
  }
  __syncthreads();
}

// The first token whose running count or weight reaches target (1 .. the whole): found
// (its ~key and index) and found_w (the running weight with it).
template <typename T>
__device__ void select(Lds& s, const RowOf<T>& row, const Weights& x, bool by_count, u64 target) {
  locate(s, 0, by_count, target);
  const int bin = s.bin;
  u64 base_n = s.base_n, base_w = s.base_w;
  if (s.in_bin <= kList) {
    rank(s, row, x, [&](double y, uint32_t) { return x.bin(y) == bin; }, by_count, target, base_n,
         base_w);
    return;
  }
  if (threadIdx.x == 0) s.lo = ~0u, s.hi = 0;
  __syncthreads();
  uint32_t mn = ~0u, mx = 0;
  row.each([&](float l, int) {
    const double y = x.log2w(l);
    if (!x.counts(y) || x.bin(y) != bin) return;
    const uint32_t key = key_of(l);
    mn = key < mn ? key : mn;
    mx = key > mx ? key : mx;
  });
  atomicMin(&s.lo, mn);
  atomicMax(&s.hi, mx);
  __syncthreads();
  uint32_t lo = s.lo, hi = s.hi;
  while (lo != hi) {
    int shift = 0;
    while ((hi - lo) >> shift >= (uint32_t)kBins) ++shift;
    for (int j = threadIdx.x; j < kBins; j += kThreads) s.count[1][j] = 0, s.weight[1][j] = 0;
    __syncthreads();
    row.each([&](float l, int) {
      const uint32_t key = key_of(l);
      if (key < lo || key > hi) return;
      const u64 units = x.units(x.weight(x.log2w(l)));
      if (units == 0) return;
      atomicAdd(&s.count[1][(hi - key) >> shift], 1);
      atomicAdd(&s.weight[1][(hi - key) >> shift], units);
    });
    __syncthreads();
    scan(s, 1);
    locate(s, 1, by_count, by_count ? target - base_n : target - base_w);
    const uint32_t j = s.bin;
    base_n += s.base_n, base_w += s.base_w;
    const uint32_t above = hi - (j << shift), width = (1u << shift) - 1;
    hi = above;
    lo = above - lo > width ? above - width : lo;
    const int n = s.in_bin;
    __syncthreads();
    if (n <= kList) {
      rank(s, row, x, [&](double, uint32_t key) { return key >= lo && key <= hi; }, by_count,
           target, base_n, base_w);
      return;
    }
  }
  // one value: its tokens weigh the same
  const u64 each = x.units(x.weight(x.log2w(value_of(lo))));
  const u64 j = by_count ? target - base_n : (target - base_w + each - 1) / each;
  nth(s, row, lo, j);
  if (threadIdx.x == 0) s.found_w = base_w + j * each;
  __syncthreads();
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Lds s;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
  const RowOf<T> row((const T*)a.logits + b * a.stride, a.V);
  if (tid < 64) s.table[tid] = exp2(tid / 64.0);
  // the largest, at its lowest index
  u64 best = 0;
  row.each([&](float l, int i) {
    const uint32_t key = key_of(l);
    const u64 v = (u64)key << 32 | ~(uint32_t)i;
    if (key && v > best) best = v;
  });
  for (int d = 1; d < 64; d *= 2) {
    const u64 o = shfl_xor64(best, d);
    best = o > best ? o : best;
  }
  if (lane == 0) s.wave_w[wave] = best;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) best = s.wave_w[w] > best ? s.wave_w[w] : best;
  const float t = a.temperature ? a.temperature[b] : 1.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  if (best == 0 || !(t > 0.0f) || k == 1) {
    if (tid == 0) {
      a.tokens[b] = best == 0 ? -1 : (int32_t)~(uint32_t)best;
      if (a.probs) a.probs[b] = best == 0 ? 0.0f : 1.0f;
    }
    return;
  }
  Weights x;
  x.table = s.table;
  x.top = value_of((uint32_t)(best >> 32));
  x.per = 1.4426950408889634 / (double)t;
  x.frac = a.frac;
  x.bins = (double)kBins / (double)(a.frac + 1);
  for (int j = tid; j < kBins; j += kThreads) s.count[0][j] = 0, s.weight[0][j] = 0;
  const float floor_p = a.min_p ? a.min_p[b] : 0.0f;
  const double least = floor_p > 0.0f ? floor_p < 1.0f ? (double)floor_p : 1.0 : 0.0;
  u64 above = 0;  // of what min-p keeps
  __syncthreads();
  row.each([&](float l, int) {
    const double y = x.log2w(l);
    if (!x.counts(y)) return;
    const double w = x.weight(y);
    const u64 units = x.units(w);
    if (units == 0) return;
    const int j = x.bin(y);
    atomicAdd(&s.count[0][j], 1);
    atomicAdd(&s.weight[0][j], units);
    if (w >= least) above += units;
  });
  for (int d = 1; d < 64; d *= 2) above += shfl_xor64(above, d);
  __syncthreads();
  scan(s, 0);
  // what min-p keeps
  if (lane == 0) s.wave_w[wave] = above;
  __syncthreads();
  u64 enough = 0;
  for (int w = 0; w < kWaves; ++w) enough += s.wave_w[w];
  // top-k, top-p and the token, in turn
  u64 kept = s.weight[0][kBins - 1];
  const float p = a.top_p ? a.top_p[b] : 1.0f, u = a.u[b];
  for (int ask = 0; ask < 3; ++ask) {
    u64 target;
    if (ask == 0) {
      if (k <= 0 || k >= s.count[0][kBins - 1]) continue;
      target = k;
    } else if (ask == 1) {
      if (!(p < 1.0f)) continue;
      const double to = ceil((double)(p > 0.0f ? p : 0.0f) * (double)kept);
      target = to < 1.0 ? 1 : (u64)to;
    } else {
      kept = enough < kept ? enough : kept;
      target = u > 0.0f ? (u64)((double)(u < 1.0f ? u : 1.0f) * (double)kept) + 1 : 1;
    }
    if (ask > 0 && target > kept) target = kept;
    select(s, row, x, ask == 0, target);
    if (ask < 2) kept = s.found_w;
  }
  if (tid == 0) {
    a.tokens[b] = (int32_t)(uint32_t)s.found;
    if (a.probs) {
      const double w = x.weight(x.log2w(value_of(~(uint32_t)(s.found >> 32))));
      a.probs[b] = (float)(w * __builtin_bit_cast(double, (uint64_t)(1023 + a.frac) << 52) /
                           (double)kept);
    }
  }
}

}  // namespace

hipError_t launch_sample(const void* logits, d2moe_dtype dtype, int64_t stride, int B, int V,
                         const float* u, const float* temperature, const int32_t* top_k,
                         const float* top_p, const float* min_p, int32_t* tokens, float* probs,
                         hipStream_t s) {
  if (B == 0) return hipSuccess;
  int bits = 0;
  while ((1 << bits) < V) ++bits;
  SampleArgs a{logits, stride, V, 62 - bits < 51 ? 62 - bits : 51, u, temperature, top_k, top_p,
               min_p, tokens, probs};
  if (dtype == D2MOE_BF16)
    sample_kernel<uint16_t><<<B, kThreads, 0, s>>>(a);
  else
    sample_kernel<float><<<B, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace d2moe
