// One token per row of logits, by temperature, top-k, top-p, min-p and a given random
// number.  With w_i = exp((l_i - max l) / t) and the tokens in descending order of l
// (ties: ascending index), every bound keeps a beginning of that order, so the kept
// tokens are one, of weight W = the least of the bounds' sums; the token is the first
// whose running sum passes u W.  All of it is one question, asked up to three times:
// the first token whose running count or sum reaches a target.
//
// No row is sorted.  Where top-k or min-p leave few tokens, those are listed, sorted and
// summed: they lie above the k-th largest of the threads' own maxima, which k tokens at
// least reach, or above min-p.  Otherwise a histogram over log2 w, of weights and where
// asked counts, says in which of 2048 bins the target lies, and only that bin's tokens,
// some dozens, are listed; a bin with more than fit is divided by its keys until they
// fit or are all equal.
//
// Weights are integers, w in units of 2^-frac, as small as V of them leave room for
// in 64 bits (2^-47 at 32000 tokens).  Their sums are exact, so that no order of
// additions turns a choice; a token below half a unit is never drawn.
//
// Bound by the instructions of the one CU that has a row: 28 a token for its weight in a
// sum, 36 with its bin, 5 for a list.  (One row of 32000 in binary32 with top-p: 20 to 23
// us, by what the settings leave, of which 9 in the histogram; 256 of 131072 in bf16 with
// all bounds: 71 to 75 us, reading them alone 11; the rows without top-k take longest, 37 us
// of it for the histogram's pass, one over four loads ahead no less.)  512 threads a row
// were slower, 27 and 96 us.
#include <cfloat>

#include "decoder.h"

namespace d2moe {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2 * kThreads, kList = 512;
constexpr int kSteps = 256;     // of the table of powers, a unit of log2
constexpr int kBinSteps = 4;    // of a bin: 32 units in all, the last bin takes what is below

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

// A row by kThreads threads, 16 bytes a thread at a time.
__device__ inline float load1(const float* p) { return *p; }
__device__ inline float load1(const uint16_t* p) { return bf2f(*p); }
template <typename T>
struct RowOf {
  static constexpr int PER = 16 / sizeof(T), HELD = 16;
  const T* p;
  int V, head, chunks;  // elements before the first whole 16 bytes; those whole ones
  __device__ RowOf(const T* row, int V) : p(row), V(V) {
    head = (int)((16 - ((uintptr_t)row & 15)) % 16 / sizeof(T));
    head = head < V ? head : V;
    chunks = (V - head) / PER;
  }
  __device__ static float value(const uint4& x, int e) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    if constexpr (sizeof(T) == 4)
      return __uint_as_float(w[e]);
    else
      return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
  }
  __device__ uint4 load(int c) const {
    return *(const uint4*)(p + head + (int64_t)(c < chunks ? c : 0) * PER);
  }
  // f(value, index) of this thread's element at the ends, if it has one
  template <typename F>
  __device__ void ends(F f) const {
    if ((int)threadIdx.x >= V - chunks * PER) return;
    const int i = (int)threadIdx.x < head ? threadIdx.x : threadIdx.x + chunks * PER;
    f(load1(p + i), i);
  }
  // f(16 bytes, index of the first) of the others, four loaded together
  template <typename F>
  __device__ void body(F f) const {
    for (int c0 = threadIdx.x; c0 < chunks; c0 += 4 * kThreads) {
      uint4 x[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = load(c0 + j * kThreads);
#pragma unroll 1
      for (int c = c0; c < chunks && c < c0 + 4 * kThreads; c += kThreads) {
        f(x[0], head + c * PER);
        x[0] = x[1], x[1] = x[2], x[2] = x[3];
      }
    }
  }
  // f(four values) for all of them, -infinity for what is missing
  template <typename F>
  __device__ void fours(F f) const {
    float one[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    ends([&](float l, int) { one[0] = l; });
    f(one);
    body([&](const uint4& y, int) {
      if constexpr (sizeof(T) == 4) {
        const float l[4] = {value(y, 0), value(y, 1), value(y, 2), value(y, 3)};
        f(l);
      } else {
        uint4 r = y;
#pragma unroll 1
        for (int h = 0; h < PER / 4; ++h) {
          const float l[4] = {value(r, 0), value(r, 1), value(r, 2), value(r, 3)};
          f(l);
          r.x = r.z, r.y = r.w;
        }
      }
    });
  }
  // f(value, index) of the wanted values among 16 bytes, seldom any
  template <typename W, typename F>
  __device__ static void pick(uint4 x, int i0, W want, F f) {
    uint32_t in = 0;
#pragma unroll
    for (int e = 0; e < PER; ++e) in |= want(value(x, e)) ? 1u << e : 0;
    while (in) {
      const int e = __ffs(in) - 1;
      in &= in - 1;
      const int bit = 8 * (int)sizeof(T) * e;
      const uint64_t two = bit & 64 ? (uint64_t)x.w << 32 | x.z : (uint64_t)x.y << 32 | x.x;
      const uint32_t one = (uint32_t)(two >> (bit & 63));
      f(__uint_as_float(sizeof(T) == 4 ? one : one << 16), i0 + e);
    }
  }
  template <typename W, typename F>
  __device__ void each(W want, F f) const {
    ends([&](float l, int i) {
      if (want(l)) f(l, i);
    });
    body([&](const uint4& x, int i0) { pick(x, i0, want, f); });
  }
  template <typename F>
  __device__ void each_in(float lo, float hi, F f) const {
    each([=](float l) { return l >= lo && l <= hi; }, f);
  }
};

// Weights of a row: log2 w = (l - top) per, and 2^it by a table of 2^(i / 256) and the
// series of 2^r, |r| <= 1/512, to the third power (the next term is 2^-42 of the whole,
// alike for all tokens and 0 for the largest).
struct Weights {
  const double* table;
  double top, per;  // per = 1 / (t ln 2)
  int frac;
  struct At {
    double y, n;
    int step;  // n, the nearest of kSteps a unit
  };
  // (NaN and what is far below half a unit: a quarter of one, which is none)
  __device__ double log2w(float l) const {
    return fmax(((double)l - top) * per, -(double)(frac + 2));
  }
  __device__ At at(double y) const {
    constexpr double kShift = 6755399441055744.0;  // 1.5 2^52: whole numbers in the last bits
    const double s = fma(y, (double)kSteps, kShift);
    return At{y, s - kShift, (int)(uint32_t)__builtin_bit_cast(uint64_t, s)};
  }
  __device__ int bin(const At& a) const {
    const int b = (uint32_t)-a.step / kBinSteps;
    return b < kBins ? b : kBins - 1;
  }
  __device__ double scaled(const At& a, int shift) const {  // w 2^shift
    const double r = fma(a.n, -1.0 / kSteps, a.y);
    double s = fma(r, 0.055504108664821576, 0.2402265069591007);  // (ln 2)^3 / 3!, and so on
    s = fma(s, r, 0.6931471805599453);
    s = fma(s, r, 1.0) * table[a.step & (kSteps - 1)];
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    const uint32_t hi = (uint32_t)(u >> 32) + ((uint32_t)((a.step >> 8) + shift) << 20);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)u);
  }
  __device__ double weight(const At& a) const { return scaled(a, frac); }
  __device__ static uint64_t units(double w) {  // rounded to nearest
    return __builtin_bit_cast(uint64_t, w + 4503599627370496.0) & 0xfffffffffffffull;
  }
  // values that may lie in a bin, and a little more
  __device__ void range(int bin, float& lo, float& hi) const {
    const double a = top - (kBinSteps * (bin + 1) + 1) / (kSteps * per);
    const double b = top - (kBinSteps * bin - 1) / (kSteps * per);
    lo = (float)(a - 1e-6 * fabs(a) - 1e-37);
    hi = (float)(b + 1e-6 * fabs(b) + 1e-37);
    if (!(lo <= hi)) lo = -INFINITY, hi = INFINITY;  // (1 / t is 0)
    // -infinity is in no range: it is never drawn, and its key 0 stands for no value
    lo = bin == kBins - 1 ? -FLT_MAX : fmaxf(lo, -FLT_MAX);
  }
};
static_assert(kSteps == 256, "scaled() takes units by a shift of 8");

typedef unsigned long long u64;

struct Lds {
  double table[kSteps];
  u64 weight[kBins];
  int count[kBins];
  // a list: ~key and index, weight; sorted, with the running sums
  u64 order[kList], units[kList], sorted[kList], sums[kList];
  int place[kList];
  u64 part[2][kWaves];
  int n, bin;
  u64 base_n, base_w, end_w, found, found_w;
};

template <int CTRL>
__device__ inline u64 row_shift(u64 v) {  // 0 where the row of 16 lanes ends
  const uint32_t a = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, 0xf, 0xf, true);
  const uint32_t b = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, 0xf, 0xf, true);
  return (u64)b << 32 | a;
}
__device__ inline u64 lane_value(u64 v, int lane) {  // lane uniform
  const uint32_t a = __builtin_amdgcn_readlane((int)(uint32_t)v, lane);
  const uint32_t b = __builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane);
  return (u64)b << 32 | a;
}
__device__ inline u64 row_scan(u64 v) {  // running sums within 16 lanes
  v += row_shift<0x111>(v);
  v += row_shift<0x112>(v);
  v += row_shift<0x114>(v);
  v += row_shift<0x118>(v);
  return v;
}
__device__ inline u64 wave_scan(u64 v) {
  v = row_scan(v);
  const u64 a = lane_value(v, 15), b = lane_value(v, 31), c = lane_value(v, 47);
  const int row = (threadIdx.x & 63) >> 4;
  return v + (row > 0 ? a : 0) + (row > 1 ? b : 0) + (row > 2 ? c : 0);
}
// Running sums over the workgroup, and the whole.  `turn` alternates between calls, so
// that one barrier is enough.
__device__ inline u64 block_scan(Lds& s, u64 v, int& turn, u64& all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  v = wave_scan(v);
  if (lane == 63) s.part[turn][wave] = v;
  __syncthreads();
  const u64 w = row_scan(s.part[turn][lane & (kWaves - 1)]);
  turn ^= 1;
  all = lane_value(w, kWaves - 1);
  return v + (wave > 0 ? lane_value(w, wave - 1) : 0);
}
__device__ inline u64 block_sum(Lds& s, u64 v, int& turn) {
  u64 all;
  block_scan(s, v, turn, all);
  return all;
}
// The largest of the keys.
__device__ inline uint32_t block_max(Lds& s, uint32_t v, int& turn) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto row_max = [](uint32_t x) {
    auto up = [](uint32_t y, uint32_t z) { return y > z ? y : z; };
    x = up(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));
    x = up(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));
    x = up(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));
    return up(x, __builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));
  };
  v = row_max(v);
  uint32_t top = 0;
#pragma unroll
  for (int r = 15; r < 64; r += 16) {
    const uint32_t o = __builtin_amdgcn_readlane((int)v, r);
    top = o > top ? o : top;
  }
  if (lane == 0) s.part[turn][wave] = top;
  __syncthreads();
  top = row_max((uint32_t)s.part[turn][lane & (kWaves - 1)]);
  turn ^= 1;
  return __builtin_amdgcn_readlane((int)top, kWaves - 1);
}

// The bins b0 .. b1 and b2.
struct Bins {
  int b0, b1, b2;
  __device__ bool has(int b) const { return (b >= b0 && b <= b1) || b == b2; }
};

__device__ constexpr Bins kAll{0, kBins, 0};

// Sorts the list's n entries (by counting those before each), weighs them and sums the
// weights up: sorted and sums.  Entries outside `bins` go to the end; the number of the
// others is returned.
__device__ int sort_list(Lds& s, const Weights& x, int n, const Bins& bins) {
  const int tid = threadIdx.x;
  if (tid < n) {
    const u64 o = s.order[tid];
    const Weights::At at = x.at(x.log2w(value_of(~(uint32_t)(o >> 32))));
    const bool in = bins.has(x.bin(at));
    s.units[tid] = in ? x.units(x.weight(at)) : 0;
    if (!in) s.order[tid] = o | ~0ull << 32;  // after every key
    s.place[tid] = 0;
  }
  __syncthreads();
  int wide = 64;  // entries a round of threads, kThreads / wide of them share one's count
  while (wide < n) wide *= 2;
  const int i = tid & (wide - 1), parts = kThreads / wide, part = tid / wide;
  if (i < n) {
    const u64 mine = s.order[i];
    const int each = (n + parts - 1) / parts, to = (part + 1) * each < n ? (part + 1) * each : n;
    int before = 0;
#pragma unroll 8
    for (int j = part * each; j < to; ++j) before += s.order[j] < mine;
    if (before) atomicAdd(&s.place[i], before);
  }
  __syncthreads();
  if (tid < n) {
    const int at = s.place[tid];
    s.sorted[at] = s.order[tid];
    s.sums[at] = s.units[tid];
  }
  __syncthreads();
  if (tid < 64) {  // one wave sums them up, kList / 64 neighbours a lane
    constexpr int kEach = kList / 64;
    u64 v[kEach], run = 0;
    int in = 0;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int j = tid * kEach + e;
      v[e] = run += j < n ? s.sums[j] : 0;
      in += j < n && s.sorted[j] >> 32 != 0xffffffffu;
    }
    const u64 from = wave_scan(run) - run;
#pragma unroll
    for (int e = 0; e < kEach; ++e) s.sums[tid * kEach + e] = from + v[e];
    const int all = (int)wave_scan(in);
    if (tid == 63) s.n = all;
  }
  __syncthreads();
  return s.n;
}

// A thread's two bins of the histogram with the sums before them.
struct Prefix {
  u64 w, w0, w1, n, n0, n1;  // before; of its two bins
  u64 all_w, all_n;
};
__device__ void prefix_of(Lds& s, Prefix& p, bool counts, int& turn) {
  const int j = 2 * threadIdx.x;
  p.w0 = s.weight[j], p.w1 = s.weight[j + 1];
  p.w = block_scan(s, p.w0 + p.w1, turn, p.all_w) - p.w0 - p.w1;
  p.n = p.n0 = p.n1 = p.all_n = 0;
  if (!counts) return;
  p.n0 = s.count[j], p.n1 = s.count[j + 1];
  p.n = block_scan(s, p.n0 + p.n1, turn, p.all_n) - p.n0 - p.n1;
}
// The bin whose running count (by_count) or weight is the first to reach target, base_n
// and base_w the sums before it, end_w that with it; the list is empty then.
__device__ void locate(Lds& s, const Prefix& p, bool by_count, u64 target) {
  const u64 a = by_count ? p.n : p.w, b = a + (by_count ? p.n0 : p.w0);
  const u64 c = b + (by_count ? p.n1 : p.w1);
  if (a < target && target <= c) {
    const bool second = target > b;
    s.bin = 2 * threadIdx.x + second;
    s.base_n = p.n + (second ? p.n0 : 0);
    s.base_w = p.w + (second ? p.w0 : 0);
    s.end_w = s.base_w + (second ? p.w1 : p.w0);
  }
  if (threadIdx.x == 0) s.n = 0;
  __syncthreads();
}

// One more entry of the list, if there is room.
__device__ inline void append(Lds& s, float l, int i) {
  const int to = atomicAdd(&s.n, 1);
  if (to < kList) s.order[to] = (u64)~key_of(l) << 32 | (uint32_t)i;
}

// Of the listed tokens (in `bins`), the first whose running count or weight reaches target,
// base_n and base_w before the first.  False: there are more than the list holds.
__device__ bool pick(Lds& s, const Weights& x, const Bins& bins, bool by_count, u64 target,
                     u64 base_n, u64 base_w) {
  __syncthreads();
  if (s.n > kList) return false;
  const int n = sort_list(s, x, s.n, bins), i = threadIdx.x;
  if (i < n) {
    const u64 run = by_count ? base_n + i + 1 : base_w + s.sums[i];
    const u64 was = by_count ? run - 1 : i ? base_w + s.sums[i - 1] : base_w;
    if (was < target && target <= run) {
      s.found = s.sorted[i];
      s.found_w = base_w + s.sums[i];
    }
  }
  __syncthreads();
  return true;
}

// The j-th token in index order, from 1, of one key.
template <typename T>
__device__ void nth(Lds& s, const RowOf<T>& row, uint32_t key, u64 j, int& turn) {
  u64 before = 0;
  for (int i0 = 0; i0 < row.V && before < j; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const u64 mine = i < row.V && key_of(load1(row.p + i)) == key;
    u64 all;
    const u64 run = before + block_scan(s, mine, turn, all);
    if (mine && run == j) s.found = (u64)~key << 32 | (uint32_t)i;
    before += all;
  }
  __syncthreads();
}

// The first token whose running count or weight reaches target; p: the histogram's
// sums.  found is its ~key and index, found_w the running weight with it.  (A division
// by keys uses the histogram's memory, but not p.)
template <typename T>
__device__ void select(Lds& s, const RowOf<T>& row, const Weights& x, const Prefix& p, bool by_count,
                       u64 target, int& turn) {
  locate(s, p, by_count, target);
  const int bin = s.bin;
  u64 base_n = s.base_n, base_w = s.base_w;
  float least, most;
  x.range(bin, least, most);
  row.each_in(least, most, [&](float l, int i) { append(s, l, i); });
  if (pick(s, x, Bins{bin, bin, bin}, by_count, target, base_n, base_w)) return;
  // by keys, from the bin's least and largest one on
  uint32_t mn = 0, mx = 0;
  row.each_in(least, most, [&](float l, int) {
    if (x.bin(x.at(x.log2w(l))) != bin) return;
    const uint32_t key = key_of(l);
    mn = ~key > mn ? ~key : mn;
    mx = key > mx ? key : mx;
  });
  uint32_t lo = ~block_max(s, mn, turn), hi = block_max(s, mx, turn);
  // (each time 2^11 times fewer keys: three times at most)
  for (int round = 0; lo != hi && round < 3; ++round) {
    int shift = 0;
    while ((hi - lo) >> shift >= (uint32_t)kBins) ++shift;
    for (int j = threadIdx.x; j < kBins; j += kThreads) s.count[j] = 0, s.weight[j] = 0;
    __syncthreads();
    row.each_in(value_of(lo), value_of(hi), [&](float l, int) {
      const uint32_t j = (hi - key_of(l)) >> shift;
      atomicAdd(&s.count[j], 1);
      atomicAdd(&s.weight[j], x.units(x.weight(x.at(x.log2w(l)))));
    });
    __syncthreads();
    Prefix q;
    prefix_of(s, q, true, turn);
    locate(s, q, by_count, by_count ? target - base_n : target - base_w);
    const uint32_t j = s.bin;
    base_n += s.base_n, base_w += s.base_w;
    const uint32_t above = hi - (j << shift), width = (1u << shift) - 1;
    hi = above;
    lo = above - lo > width ? above - width : lo;
    row.each_in(value_of(lo), value_of(hi), [&](float l, int i) { append(s, l, i); });
    if (pick(s, x, kAll, by_count, target, base_n, base_w)) return;
  }
  // one value: its tokens weigh the same
  const u64 one = x.units(x.weight(x.at(x.log2w(value_of(lo)))));
  const u64 j = by_count ? target - base_n : (target - base_w + one - 1) / one;
  nth(s, row, lo, j, turn);
  if (threadIdx.x == 0) s.found_w = base_w + j * one;
  __syncthreads();
}

// The weights, and where asked the counts, of the tokens from `from` on by bins; `above`:
// the weight of those of `least` units and more.  ALL: every token, no counts, no least.
// Four tokens at a time, so that what one waits for passes under the others.
template <typename T, bool ALL>
__device__ void histogram(Lds& s, const RowOf<T>& row, const Weights& x, float from, double least,
                          bool counts, u64& above) {
  for (int j = threadIdx.x; j < kBins; j += kThreads) s.count[j] = 0, s.weight[j] = 0;
  u64 rest = 0;  // of the last bin, which many may share
  int rest_n = 0;
  __syncthreads();
  row.fours([&](const float (&l)[4]) {
    Weights::At at[4];
    double w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) at[e] = x.at(x.log2w(l[e]));
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = x.weight(at[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const u64 units = x.units(w[e]);
      const int bin = x.bin(at[e]);
      if constexpr (!ALL) {
        if (units == 0 || l[e] < from) continue;
        if (w[e] >= least) above += units;
      }
      if (bin == kBins - 1) {
        rest += units, ++rest_n;
      } else {
        atomicAdd(&s.weight[bin], units);
        if (!ALL && counts) atomicAdd(&s.count[bin], 1);
      }
    }
  });
  if (rest > 0) {
    atomicAdd(&s.weight[kBins - 1], rest);
    if (!ALL && counts) atomicAdd(&s.count[kBins - 1], rest_n);
  }
  __syncthreads();
}
// The weight of all tokens.
template <typename T>
__device__ u64 whole_sum(Lds& s, const RowOf<T>& row, const Weights& x, int& turn) {
  u64 sum = 0;
  row.fours([&](const float (&l)[4]) {
    Weights::At at[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) at[e] = x.at(x.log2w(l[e]));
#pragma unroll
    for (int e = 0; e < 4; ++e) sum += x.units(x.weight(at[e]));
  });
  return block_sum(s, sum, turn);
}

// The target that the first token past top-p's part of a sum, or past u of it, reaches.
__device__ inline u64 top_p_target(float p, u64 sum) {
  const double at = ceil((double)(p > 0.0f ? p : 0.0f) * (double)sum);
  const u64 target = at < 1.0 ? 1 : (u64)at;
  return target < sum ? target : sum;
}
__device__ inline u64 token_target(float u, u64 sum) {
  const u64 at = u > 0.0f ? (u64)((double)(u < 1.0f ? u : 1.0f) * (double)sum) + 1 : 1;
  return at < sum ? at : sum;
}

// Top-p and the token in one pass over the row: the bin in which top-p's sum ends bounds
// the kept sum (`above` at most, what min-p keeps), so the token's bins are known as well.
// found is its ~key and index, kept the sum.  False: the bins hold more than a list.
template <typename T>
__device__ bool select_both(Lds& s, const RowOf<T>& row, const Weights& x, const Prefix& p,
                            u64 target, float u, u64 above, u64& kept) {
  auto least_of = [](u64 a, u64 b) { return a < b ? a : b; };
  locate(s, p, false, target);
  Bins bins;
  bins.b2 = s.bin;
  const u64 base_p = s.base_w, most = least_of(above, s.end_w);
  __syncthreads();
  locate(s, p, false, token_target(u, least_of(above, target)));
  bins.b0 = s.bin;
  const u64 base_u = s.base_w;
  __syncthreads();
  locate(s, p, false, token_target(u, most));
  bins.b1 = s.bin;
  float lo_u, hi_u, lo_p, hi_p, unused;
  x.range(bins.b0, unused, hi_u);
  x.range(bins.b1, lo_u, unused);
  x.range(bins.b2, lo_p, hi_p);
  row.each([=](float l) { return (l >= lo_u && l <= hi_u) || (l >= lo_p && l <= hi_p); },
           [&](float l, int i) { append(s, l, i); });
  __syncthreads();
  if (s.n > kList) {
    __syncthreads();  // every wave has seen it: the caller's next search empties the list
    return false;
  }
  const int n = sort_list(s, x, s.n, bins), i = threadIdx.x;
  // the token's bins come first; the others' sums begin anew where they do not adjoin
  const u64 run = i < n ? s.sums[i] : 0, was = i < n && i > 0 ? s.sums[i - 1] : 0;
  const bool first =
      i < n && x.bin(x.at(x.log2w(value_of(~(uint32_t)(s.sorted[i] >> 32))))) <= bins.b1;
  if (first && (i + 1 == n || x.bin(x.at(x.log2w(value_of(~(uint32_t)(s.sorted[i + 1] >> 32))))) >
                                  bins.b1))
    s.end_w = run;  // of the token's bins
  __syncthreads();
  const u64 base = bins.b2 <= bins.b1 ? base_u : first ? ~0ull : base_p - s.end_w;
  if (i < n && base != ~0ull && base + was < target && target <= base + run)
    s.found_w = base + run;
  __syncthreads();
  kept = least_of(above, s.found_w);
  const u64 to = token_target(u, kept);
  if (first && base_u + was < to && to <= base_u + run) s.found = s.sorted[i];
  __syncthreads();
  return true;
}

// A key that k tokens of the row at least reach: the threads' maxima (`mine`, 0: none) in
// bins from the largest down, then the least of those in the first bins that hold k.
// 0 where the threads are too few.
__device__ uint32_t cut_of(Lds& s, uint32_t mine, uint32_t top, int k, int& turn) {
  const uint32_t least = ~block_max(s, mine ? ~mine : 0, turn);
  for (int j = threadIdx.x; j < kBins; j += kThreads) s.weight[j] = 0;
  __syncthreads();
  int shift = 0;
  while ((top - least) >> shift >= (uint32_t)kBins) ++shift;
  const uint32_t bin = (top - mine) >> shift;
  if (mine) atomicAdd(&s.weight[bin], 1ull);
  __syncthreads();
  Prefix p;
  prefix_of(s, p, false, turn);
  if (p.all_w < (u64)k) return 0;
  locate(s, p, false, k);
  return ~block_max(s, mine && bin <= (uint32_t)s.bin ? ~mine : 0, turn);
}

// HELD: the row is read once into registers for the largest value and for the list.
template <typename T, bool HELD>
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleArgs a) {
  __shared__ Lds s;
  const int tid = threadIdx.x, b = blockIdx.x;
  const RowOf<T> row((const T*)a.logits + b * a.stride, a.V);
  constexpr int PER = RowOf<T>::PER, N = HELD ? RowOf<T>::HELD : 1;
  uint4 held[N];
  if constexpr (HELD) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j * kThreads < row.chunks) held[j] = row.load(j * kThreads + tid);
  }
  const float t = a.temperature ? a.temperature[b] : 1.0f;
  const int k = a.top_k ? a.top_k[b] : 0;
  const float p = a.top_p ? a.top_p[b] : 1.0f, u = a.u[b];
  const float floor_p = a.min_p ? a.min_p[b] : 0.0f;
  const bool whole = p < 1.0f;  // the sum of what top-k leaves is asked for
  int turn = 0;
  if (tid < kSteps) s.table[tid] = exp2(tid / (double)kSteps);
  if (tid == 0) s.n = 0;
  float largest = -INFINITY;
  auto more = [&](const uint4& x) {
#pragma unroll
    for (int e = 0; e < PER; ++e) largest = fmaxf(largest, row.value(x, e));
  };
  row.ends([&](float l, int) { largest = fmaxf(largest, l); });
  if constexpr (HELD) {
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j * kThreads + tid < row.chunks) more(held[j]);
  } else {
    row.body([&](const uint4& x, int) { more(x); });
  }
  const uint32_t mine = key_of(largest), top = block_max(s, mine, turn);
  const float top_l = value_of(top);
  if (top == 0) {
    if (tid == 0) {
      a.tokens[b] = -1;
      if (a.probs) a.probs[b] = 0.0f;
    }
    return;
  }
  if (!(t > 0.0f) || k == 1 || top_l == INFINITY) {
    // the first of the largest; of infinite ones, which share the whole, one in its turn
    u64 n = 1, j = 1;
    if (t > 0.0f && k != 1) {
      u64 mine_n = 0;
      row.each_in(top_l, top_l, [&](float, int) { ++mine_n; });
      n = block_sum(s, mine_n, turn);
      n = k > 0 && (u64)k < n ? k : n;
      n = whole ? top_p_target(p, n) : n;
      j = token_target(u, n);
    }
    if (j == 1) {
      uint32_t first = 0;  // ~index
      row.each_in(top_l, top_l, [&](float, int i) {
        first = ~(uint32_t)i > first ? ~(uint32_t)i : first;
      });
      first = block_max(s, first, turn);
      if (tid == 0) s.found = ~first;
    } else {
      nth(s, row, top, j, turn);
    }
    if (tid == 0) {
      a.tokens[b] = (int32_t)(uint32_t)s.found;
      if (a.probs) a.probs[b] = (float)(1.0 / (double)n);
    }
    return;
  }
  Weights x;
  x.table = s.table;
  x.top = (double)top_l;
  x.per = 1.4426950408889634 / (double)t;
  x.frac = a.frac;
  const double least = (floor_p > 0.0f ? floor_p < 1.0f ? (double)floor_p : 1.0 : 0.0) *
                       (double)(1ull << a.frac);
  float from = -INFINITY;  // below: not kept
  if (k > 0 && k <= kList) {
    const uint32_t cut = cut_of(s, mine, top, k, turn);
    if (cut) from = value_of(cut);
  }
  if (least > 0.0 && (!whole || k <= 0)) {  // (a little lower than min-p)
    const double bound = floor_p < 1.0f ? log2((double)floor_p) : 0.0;
    const float f = (float)(x.top + (bound - 1e-3) / x.per);
    from = fmaxf(from, f - 1e-6f * fabsf(f) - 1e-37f);
  }
  u64 kept = 0, found = 0;
  bool listed = false;
  if (from > -INFINITY || a.V <= kList) {
    auto list = [&](float l, int i) { append(s, l, i); };
    if (tid == 0) s.n = 0;
    __syncthreads();
    if constexpr (HELD) {
      row.ends([&](float l, int i) {
        if (l >= from) list(l, i);
      });
#pragma unroll
      for (int j = 0; j < N; ++j) {
        if (j % 4 == 2 && *(volatile int*)&s.n > kList) break;  // they do not fit
        if (j * kThreads + tid < row.chunks)
          row.pick(held[j], row.head + (j * kThreads + tid) * PER,
                   [=](float l) { return l >= from; }, list);
      }
    } else {
      row.each_in(from, top_l, list);
    }
    __syncthreads();
    listed = s.n <= kList;
  }
  if (listed) {
    int n = sort_list(s, x, s.n, kAll);
    n = k > 0 && k < n ? k : n;
    if (whole) {
      // (of a row cut off at min-p top-p still takes its part of everything)
      const u64 sum = k > 0 || from == -INFINITY ? s.sums[n - 1] : whole_sum(s, row, x, turn);
      const u64 target = top_p_target(p, sum);
      if (tid == 0) s.bin = n;  // (not reached within the list)
      __syncthreads();
      if (tid < n && s.sums[tid] >= target && (tid == 0 || s.sums[tid - 1] < target)) s.bin = tid + 1;
      __syncthreads();
      n = s.bin;
    }
    if (least > 0.0) {
      bool keeps = false;
      if (tid < n)
        keeps = x.weight(x.at(x.log2w(value_of(~(uint32_t)(s.sorted[tid] >> 32))))) >= least;
      n = (int)block_sum(s, keeps, turn);
    }
    kept = s.sums[n - 1];
    const u64 target = token_target(u, kept);
    if (tid < n && s.sums[tid] >= target && (tid == 0 || s.sums[tid - 1] < target))
      s.found = s.sorted[tid];
    __syncthreads();
    found = s.found;
  } else {
    u64 above = 0;  // of what min-p keeps
    if (k <= 0 && !(least > 0.0))
      histogram<T, true>(s, row, x, from, least, false, above);
    else
      histogram<T, false>(s, row, x, whole && k <= 0 ? -INFINITY : from, least, k > 0, above);
    Prefix q;
    prefix_of(s, q, k > 0, turn);
    above = least > 0.0 ? block_sum(s, above, turn) : q.all_w;
    kept = q.all_w;
    for (int ask = 0; ask < 3; ++ask) {  // top-k, top-p and the token, in turn
      u64 target;
      if (ask == 0) {
        if (k <= 0 || (u64)k >= q.all_n) continue;
        target = k;
      } else if (ask == 1) {
        if (!whole) continue;
        target = top_p_target(p, kept);
        if (select_both(s, row, x, q, target, u, above, kept)) break;
      } else {
        kept = above < kept ? above : kept;
        target = token_target(u, kept);
      }
      select(s, row, x, q, ask == 0, target, turn);
      if (ask < 2) kept = s.found_w;
    }
    found = s.found;
  }
  if (tid == 0) {
    a.tokens[b] = (int32_t)(uint32_t)found;
    if (a.probs) {
      const double w = x.weight(x.at(x.log2w(value_of(~(uint32_t)(found >> 32)))));
      a.probs[b] = (float)(w / (double)kept);
    }
  }
}

constexpr int kMostRows = 1 << 21;  // of a launch, whose threads must be fewer than 2^32

// Rows of up to 16 times 16 bytes a thread are held.
template <typename T>
hipError_t run_sample(SampleArgs a, int B, hipStream_t s) {
  for (;;) {
    const int n = B < kMostRows ? B : kMostRows;
    if (a.V <= RowOf<T>::HELD * kThreads * RowOf<T>::PER)
      sample_kernel<T, true><<<n, kThreads, 0, s>>>(a);
    else
      sample_kernel<T, false><<<n, kThreads, 0, s>>>(a);
    const hipError_t err = hipGetLastError();
    B -= n;
    if (err != hipSuccess || B == 0) return err;
    a.logits = (const T*)a.logits + n * a.stride;
    a.u += n;
    if (a.temperature) a.temperature += n;
    if (a.top_k) a.top_k += n;
    if (a.top_p) a.top_p += n;
    if (a.min_p) a.min_p += n;
    a.tokens += n;
    if (a.probs) a.probs += n;
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
  const SampleArgs a{logits, stride, V,     62 - bits < 51 ? 62 - bits : 51, u, temperature,
                     top_k,  top_p,  min_p, tokens, probs};
  return dtype == D2MOE_BF16 ? run_sample<uint16_t>(a, B, s) : run_sample<float>(a, B, s);
}

}  // namespace d2moe
