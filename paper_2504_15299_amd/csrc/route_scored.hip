// Routing by scores: softmax or sigmoid of the gate logits, experts chosen by score
// plus a bias, within the best groups of experts, weights from the scores alone;
// then bit-widths, counts, scan and permutation as route.hip leaves them.
//
// Scores and their comparisons are binary64, so that the choice is that of the
// formula wherever two scores differ by more than its last bits (binary32 would turn
// one of 40000 choices among 64 experts).  The comparisons are of integers in the same
// order, the upper words first (as binary64, 8192 tokens' choices take 11.6 us for 9.3).
//
// Up to kOneTokens tokens everything is one workgroup (16 tokens, 2 of 8 experts: 6.0
// us, latency: a load, the scores, the k maxima and seven barriers).  A wave then has up to
// four tokens one after the other, for a launch less, which counts where calls follow each
// other: 64 tokens, 2 of 8 experts, 12.3 us a call for 12.8 of two launches; 6 of 64 experts
// 9.7 at 32 tokens, 15.1 at 64, for 12.8.  (In a captured graph two are faster from 17 tokens
// on: at 16, 32 and 64 tokens, 6 of 64 experts, 7.4, 9.9 and 15.4 us, two 7.8, 7.7 and 8.0.)
// Above, a wave a token chooses, then every kBlock slots are counted, each key's counts
// scanned over the blocks, and the slots placed (up to kOneSlots by one workgroup); the
// tables between the launches lie in the part of slot_of that their block writes last.  8192
// tokens, 6 of 64 experts in 4 of 8 groups, sigmoid: 9.6 + 2.7 + 3.1 + 4.8 us, the choice
// bound by its instructions (3 MB cross the memory, 0.6 us), the others by latency.
#include "internal.h"

namespace d2moe {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kMaxKeys = 64 * 8;   // E <= 64, L <= 8
constexpr int kBlock = 1024;       // slots of a block, one a thread; the last one's up to twice
constexpr int kOneTokens = 64;     // tokens that one workgroup chooses for
constexpr int kOneSlots = 2 * kBlock - 1;  // slots that one workgroup places
constexpr int kMostTokens = 1 << 24;  // of a launch, whose threads must be fewer than 2^32
static_assert(kBlock > kMaxKeys, "a block's table fits its part of slot_of");

struct ScoredArgs {
  const float *logits, *select_bias;
  const int32_t* token_req;
  const uint8_t* bit_table;
  int T, E, k, R, b_min, b_max, L, sigmoid, groups, top_groups, renorm;
  float scale;
  int32_t* topk_idx;
  float* topk_w;
  uint8_t* topk_bits;
  int32_t *hist, *offsets, *perm, *slot_of, *flags;
  uint8_t* maxbit;
};

template <int CTRL>
__device__ inline int row_shift(int v) {  // lanes without a source keep their own
  return __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, false);
}
__device__ inline uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }
// The largest over the wave, on every lane: within rows of 16 by shifts, then over the
// rows.
__device__ inline uint32_t wave_max(uint32_t v) {
  v = larger(v, row_shift<0x111>(v));
  v = larger(v, row_shift<0x112>(v));
  v = larger(v, row_shift<0x114>(v));
  v = larger(v, row_shift<0x118>(v));
  const uint32_t a = __builtin_amdgcn_readlane(v, 15), b = __builtin_amdgcn_readlane(v, 31);
  const uint32_t c = __builtin_amdgcn_readlane(v, 47), d = __builtin_amdgcn_readlane(v, 63);
  return larger(larger(a, b), larger(c, d));
}
__device__ inline double lane_value(double v, int lane) {  // lane uniform
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t a = __builtin_amdgcn_readlane((int)(uint32_t)u, lane);
  const uint32_t b = __builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)b << 32 | a);
}
// Integers in the order of the values, neither NaN nor -0.
__device__ inline uint32_t ordered(float v) {
  const uint32_t u = __builtin_bit_cast(uint32_t, v);
  return u >> 31 ? ~u : u | 1u << 31;
}
__device__ inline uint64_t ordered(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  return u >> 63 ? ~u : u | 1ull << 63;
}
__device__ inline double wave_sum(double v) {
  for (int off = 1; off < 64; off *= 2) v += __shfl_xor(v, off, 64);
  return v;
}

// LDS between the lanes of a wave.
__device__ inline void wave_handoff() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Token t's experts by one wave, lane e with expert e; `tmp` is the wave's.  Returns
// the flag bits.  lkeys: where the slots' keys go as well.
__device__ int select(const ScoredArgs& a, int t, int lane, double (&tmp)[64], int* lkeys) {
  const bool have = lane < a.E;
  const float logit = have ? a.logits[(int64_t)t * a.E + lane] : -INFINITY;
  const double x = logit;
  int flag = 0, r = a.token_req ? a.token_req[t] : 0;
  if (r < 0 || r >= a.R) {
    flag = 2;
    r = r < 0 ? 0 : a.R - 1;
  }
  const int b = have ? a.bit_table[(int64_t)r * a.E + lane] : 0;
  double score;
  if (a.sigmoid) {
    score = 1.0 / (1.0 + exp(-x));
  } else {
    const uint32_t most = wave_max(ordered(x == x ? logit + 0.0f : -INFINITY));
    const double top = __builtin_bit_cast(float, most >> 31 ? most & ~(1u << 31) : ~most);
    const double e = x == top ? 1.0 : exp(x - top);
    const double sum = wave_sum(e == e && top > -INFINITY ? e : 0.0);
    // nothing but masked logits: no weight at all; a NaN keeps its own
    score = x == x && sum == 0.0 ? 0.0 : e / sum;
  }
  const double by = have && a.select_bias ? score + (double)a.select_bias[lane] : score;
  bool live = have;
  if (a.groups > 1) {
    // lane g sums the two best of group g, then counts the groups before it; NaN is
    // below everything
    const int size = a.E / a.groups;
    tmp[lane] = by == by ? by : -INFINITY;
    wave_handoff();
    double best = -INFINITY, next = -INFINITY;
    if (lane < a.groups)
#pragma unroll 4
      for (int i = 0; i < size; ++i) {
        const double v = tmp[lane * size + i];
        next = fmax(next, fmin(best, v));
        best = fmax(best, v);
      }
    if (size > 1) best += next;
    if (!(best == best)) best = -INFINITY;  // infinities of both signs
    wave_handoff();
    tmp[lane] = best;
    wave_handoff();
    int before = 0;
    if (lane < a.groups)
#pragma unroll 4
      for (int g = 0; g < a.groups; ++g) before += tmp[g] > best || (tmp[g] == best && g < lane);
    wave_handoff();  // the next token's group values come after
    const uint64_t on = __ballot(lane < a.groups && before < a.top_groups);
    live = have && (on >> (lane / size) & 1);
  }
  double mine = 0.0, total = 0.0;
  int idx = 0, bits = 0;
  // The largest by its upper word, by the lower one where several share that; NaN
  // comes after -infinity, what may not be chosen after that.
  const uint64_t key = by == by ? ordered(by + 0.0) : 1ull << 32;
  uint32_t upper = live ? (uint32_t)(key >> 32) : 0;
  for (int i = 0; i < a.k; ++i) {
    const uint32_t top = wave_max(upper);
    uint64_t cand = __ballot(upper == top);
    if (cand & (cand - 1)) {
      const uint32_t low = upper == top ? (uint32_t)key : 0;
      cand &= __ballot(low == wave_max(low));
    }
    const int best = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)cand) - 1);
    const double s = lane_value(score, best);
    const int bb = __builtin_amdgcn_readlane(b, best);
    if (lane == best) upper = 0;
    total += s;
    if (lane == i) mine = s, idx = best, bits = bb;
  }
  const bool out = lane < a.k && (bits < a.b_min || bits > a.b_max);
  if (__ballot(out)) flag |= 1;
  if (lane < a.k) {
    const int64_t at = (int64_t)t * a.k + lane;
    const int c = bits < a.b_min ? a.b_min : bits > a.b_max ? a.b_max : bits;
    if (a.renorm) mine = total == 0.0 ? 0.0 : mine / total;
    a.topk_idx[at] = idx;
    a.topk_bits[at] = (uint8_t)c;
    a.topk_w[at] = (float)(mine * (double)a.scale);
    if (lkeys) lkeys[at] = idx * a.L + c - a.b_min;
  }
  return flag;
}

// Many tokens, from `first` on: one wave each; the flag bits wait in perm[t].
__global__ __launch_bounds__(256) void scored_select_kernel(ScoredArgs a, int first) {
  __shared__ double tmp[4][64];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int t = first + blockIdx.x * 4 + wave;
  if (t >= a.T) return;
  const int flag = select(a, t, lane, tmp[wave], nullptr);
  if (lane == 0) a.perm[t] = flag;
}

// Exclusive scan of the keys' counts by the first wave: off[0 .. nkeys].
__device__ inline void scan_keys(const int* cnt, int* off, int nkeys, int lane) {
  constexpr int kPer = kMaxKeys / 64;
  const int per = (nkeys + 63) / 64;
  int v[kPer], sum = 0;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int j = lane * per + q;
    v[q] = q < per && j < nkeys ? cnt[j] : 0;
    sum += v[q];
  }
  int inc = sum;
  for (int d = 1; d < 64; d *= 2) {
    const int o = __shfl_up(inc, d, 64);
    if (lane >= d) inc += o;
  }
  int acc = inc - sum;
#pragma unroll
  for (int q = 0; q < kPer; ++q) {
    const int j = lane * per + q;
    if (q < per && j < nkeys) off[j] = acc;
    acc += v[q];
  }
  if (lane == 63) off[nkeys] = acc;
}

__device__ inline int key_of(const ScoredArgs& a, int s) {
  return a.topk_idx[s] * a.L + a.topk_bits[s] - a.b_min;
}

// perm and slot_of of slots first .. first + n - 1, in slot order within a key, key j's
// from base[j] on (which moves on).  mine: the key of slot first + threadIdx.x.
__device__ void place(const ScoredArgs& a, int first, int n, const int* lkeys, int mine, int* base,
                      int (&wave_cnt)[kWaves][kMaxKeys]) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nkeys = a.E * a.L;
  const uint64_t before = lane == 0 ? 0 : ~0ull >> (64 - lane);
  for (int from = 0; from < n; from += kThreads) {
    for (int j = lane; j < nkeys; j += 64) wave_cnt[wave][j] = 0;
    const bool valid = from + tid < n;
    const int s = first + from + tid;
    const int key = !valid ? 0 : from == 0 ? mine : lkeys ? lkeys[s] : key_of(a, s);
    uint64_t same = __ballot(valid);
#pragma unroll
    for (int bit = 0; bit < 9; ++bit) {
      const uint64_t m = __ballot(key >> bit & 1);
      same &= key >> bit & 1 ? m : ~m;
    }
    const int rank = __popcll(same & before);
    wave_handoff();  // (a wave's row is its own)
    if (valid && rank == 0) wave_cnt[wave][key] = __popcll(same);
    __syncthreads();
    if (valid) {
      int pos = base[key] + rank;
      for (int w = 0; w < wave; ++w) pos += wave_cnt[w][key];
      a.perm[pos] = s;
      a.slot_of[s] = pos;
    }
    if (from + kThreads >= n) break;  // nothing follows
    __syncthreads();
    for (int j = tid; j < nkeys; j += kThreads) {
      int sum = 0;
      for (int w = 0; w < kWaves; ++w) sum += wave_cnt[w][j];
      base[j] += sum;
    }
    __syncthreads();
  }
}

__device__ inline void write_totals(const ScoredArgs& a, const int* cnt, const int* off) {
  const int nkeys = a.E * a.L;
  for (int j = threadIdx.x; j <= nkeys; j += kThreads) a.offsets[j] = off[j];
  for (int e = threadIdx.x; e < a.E; e += kThreads) {
    int most = 0;
    for (int l = 0; l < a.L; ++l)
      if (cnt[e * a.L + l] > 0) most = a.b_min + l;
    a.maxbit[e] = (uint8_t)most;
  }
}

// One workgroup for all slots (kOneSlots at most), and with SELECT for the choice.
template <bool SELECT>
__global__ __launch_bounds__(kThreads) void scored_one_kernel(ScoredArgs a) {
  __shared__ double tmp[SELECT ? kWaves : 1][64];
  __shared__ int lkeys[SELECT ? kOneSlots : 1];
  __shared__ int cnt[kMaxKeys], off[kMaxKeys + 1], wave_cnt[kWaves][kMaxKeys], flag;
  const int tid = threadIdx.x, lane = tid & 63, n = a.T * a.k, nkeys = a.E * a.L;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int j = tid; j < nkeys; j += kThreads) cnt[j] = 0;
  if (tid == 0) flag = 0;
  __syncthreads();
  int fl = 0;
  if constexpr (SELECT) {
    for (int t = wave; t < a.T; t += kWaves) fl |= select(a, t, lane, tmp[wave], lkeys);
    if (lane != 0) fl = 0;
    __syncthreads();
  } else {
    for (int t = tid; t < a.T; t += kThreads) fl |= a.perm[t];
  }
  if (fl) atomicOr(&flag, fl);
  for (int s = tid; s < n; s += kThreads)
    atomicAdd(&cnt[SELECT ? lkeys[s] : key_of(a, s)], 1);
  __syncthreads();
  if (wave == 0) scan_keys(cnt, off, nkeys, lane);
  if (tid == 0) *a.flags = flag;
  __syncthreads();
  for (int j = tid; j < nkeys; j += kThreads) a.hist[j] = cnt[j];
  write_totals(a, cnt, off);
  __syncthreads();
  const int mine = tid < n ? SELECT ? lkeys[tid] : key_of(a, tid) : 0;
  place(a, 0, n, SELECT ? lkeys : nullptr, mine, off, wave_cnt);
}

// Slots of block b of nb.
__device__ inline int block_slots(const ScoredArgs& a, int b, int nb) {
  return b + 1 < nb ? kBlock : a.T * a.k - b * kBlock;
}

// Each block's counts, and its tokens' flag bits behind them.
__global__ __launch_bounds__(kThreads) void scored_count_kernel(ScoredArgs a) {
  __shared__ int cnt[kMaxKeys + 1];
  const int nkeys = a.E * a.L, first = blockIdx.x * kBlock;
  const int n = block_slots(a, blockIdx.x, gridDim.x);
  for (int j = threadIdx.x; j <= nkeys; j += kThreads) cnt[j] = 0;
  __syncthreads();
  for (int s = first + threadIdx.x; s < first + n; s += kThreads) {
    atomicAdd(&cnt[key_of(a, s)], 1);
    if (s < a.T && a.perm[s]) atomicOr(&cnt[nkeys], a.perm[s]);
  }
  __syncthreads();
  for (int j = threadIdx.x; j <= nkeys; j += kThreads) a.slot_of[first + j] = cnt[j];
}

// A wave a key: counts of the blocks to the exclusive sums, the whole to hist.
__global__ __launch_bounds__(256) void scored_scan_kernel(ScoredArgs a, int nb) {
  const int key = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int nkeys = a.E * a.L;
  if (key > nkeys) return;
  int sum = 0;
  for (int b0 = 0; b0 < nb; b0 += 64) {
    const bool in = b0 + lane < nb;
    int32_t* p = a.slot_of + (in ? b0 + lane : 0) * (int64_t)kBlock + key;
    const int v = in ? *p : 0;
    if (key == nkeys) {
      sum |= v;
      continue;
    }
    int inc = v;
    for (int d = 1; d < 64; d *= 2) {
      const int o = __shfl_up(inc, d, 64);
      if (lane >= d) inc += o;
    }
    if (in) *p = sum + inc - v;
    sum += __shfl(inc, 63, 64);
  }
  if (key == nkeys) {
    for (int d = 1; d < 64; d *= 2) sum |= __shfl_xor(sum, d, 64);
    if (lane == 0) *a.flags = sum;
  } else if (lane == 0) {
    a.hist[key] = sum;
  }
}

__global__ __launch_bounds__(kThreads) void scored_place_kernel(ScoredArgs a) {
  __shared__ int cnt[kMaxKeys], off[kMaxKeys + 1], wave_cnt[kWaves][kMaxKeys];
  const int tid = threadIdx.x, nkeys = a.E * a.L, first = blockIdx.x * kBlock;
  const int n = block_slots(a, blockIdx.x, gridDim.x);
  // everything from memory at once (a key a thread)
  const int count = tid < nkeys ? a.hist[tid] : 0;
  const int before = tid < nkeys ? a.slot_of[first + tid] : 0;
  const int mine = tid < n ? key_of(a, first + tid) : 0;
  if (tid < nkeys) cnt[tid] = count;
  __syncthreads();
  if (tid < 64) scan_keys(cnt, off, nkeys, tid);
  __syncthreads();  // and the block's part of slot_of has been read
  if (blockIdx.x == 0) {
    write_totals(a, cnt, off);
    __syncthreads();
  }
  if (tid < nkeys) off[tid] += before;
  __syncthreads();
  place(a, first, n, nullptr, mine, off, wave_cnt);
}

}  // namespace

hipError_t launch_route_scored(const void* x, d2moe_dtype xd, int T, int d, const float* Wg,
                               const float* bias, int E, int k, bool sigmoid,
                               const float* select_bias, int groups, int top_groups, bool renorm,
                               float scale, const int32_t* token_req, const uint8_t* bit_table,
                               int R, int b_min, int b_max, const d2moe_routing* out,
                               hipStream_t s) {
  const size_t row = (size_t)d * (xd == D2MOE_BF16 ? 2 : 4);
  for (int t = 0; x && t < T; t += kMostTokens) {
    const hipError_t err =
        launch_gate((const char*)x + t * row, xd, T - t < kMostTokens ? T - t : kMostTokens, d, Wg,
                    bias, E, out->logits + (int64_t)t * E, s);
    if (err != hipSuccess) return err;
  }
  ScoredArgs a{};
  a.logits = out->logits, a.select_bias = select_bias, a.token_req = token_req;
  a.bit_table = bit_table, a.T = T, a.E = E, a.k = k, a.R = R, a.b_min = b_min, a.b_max = b_max;
  a.L = b_max - b_min + 1, a.sigmoid = sigmoid, a.groups = groups, a.top_groups = top_groups;
  a.renorm = renorm, a.scale = scale, a.topk_idx = out->topk_idx, a.topk_w = out->topk_w;
  a.topk_bits = out->topk_bits, a.hist = out->hist, a.offsets = out->offsets, a.perm = out->perm;
  a.slot_of = out->slot_of, a.flags = out->flags, a.maxbit = out->expert_maxbit;
  const int n = T * k, nkeys = E * a.L;
  if (T <= kOneTokens && n <= kOneSlots) {
    scored_one_kernel<true><<<1, kThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  hipError_t err;
  for (int t = 0; t < T; t += kMostTokens) {
    const int n = T - t < kMostTokens ? T - t : kMostTokens;
    scored_select_kernel<<<(n + 3) / 4, 256, 0, s>>>(a, t);
    if ((err = hipGetLastError()) != hipSuccess) return err;
  }
  if (n <= kOneSlots) {
    scored_one_kernel<false><<<1, kThreads, 0, s>>>(a);
    return hipGetLastError();
  }
  const int nb = n / kBlock;
  scored_count_kernel<<<nb, kThreads, 0, s>>>(a);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  scored_scan_kernel<<<nkeys / 4 + 1, 256, 0, s>>>(a, nb);
  if ((err = hipGetLastError()) != hipSuccess) return err;
  scored_place_kernel<<<nb, kThreads, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace d2moe
