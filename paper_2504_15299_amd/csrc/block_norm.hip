// The norms after a block and before the next one, with the block's gate and
// the residual's scales:
//   u = post_w * y / sqrt(mean y^2 + eps),  x <- x_scale x + y_scale gate u,
//   h = pre_w * x / sqrt(mean x^2 + eps)
// One workgroup per row; the row is read once into registers (d <= 16384) and
// written once, so the kernel is bound by memory (12 bytes a value in bf16).
#include "decoder.h"

namespace d2moe {
namespace {

constexpr int kNormMax = 16384;  // columns of a row

struct NormArgs {
  float* x;
  const void *y, *gate;
  const float *post_w, *pre_w;
  void* h;
  int64_t gate_stride;
  float x_scale, y_scale, eps;
  int d;
  int64_t row0;  // of this launch
  bool y_bf, g_bf, h_bf;
};

// Rows start at multiples of an element only, which vector loads allow.
typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t h4 __attribute__((ext_vector_type(4), aligned(2)));

// Up to four consecutive values of a row of either type, n of them inside the
// row (the others become zero), one load where all four are.
__device__ inline void load_row(const void* p, bool bf, int64_t at, int n, float (&v)[4]) {
  v[0] = v[1] = v[2] = v[3] = 0.0f;
  if (n >= 4) {
    if (bf) {
      const h4 u = *(const h4*)((const uint16_t*)p + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = bf2f(u[e]);
    } else {
      const f4 f = *(const f4*)((const float*)p + at);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = f[e];
    }
  } else if (n > 0) {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) v[e] = bf ? bf2f(((const uint16_t*)p)[at + e]) : ((const float*)p)[at + e];
  }
}

// Rows that are many enough to leave the caches before they are read again are
// stored past them (1024 rows of 4096 with a gate per token: 13.4 -> 12.5 us).
template <bool PAST>
__device__ inline void store_row(void* p, bool bf, int64_t at, int n, const float (&v)[4]) {
  if (n >= 4) {
    const h4 h = {f2bf(v[0]), f2bf(v[1]), f2bf(v[2]), f2bf(v[3])};
    const f4 f = {v[0], v[1], v[2], v[3]};
    if (bf && PAST)
      __builtin_nontemporal_store(h, (h4*)((uint16_t*)p + at));
    else if (bf)
      *(h4*)((uint16_t*)p + at) = h;
    else if (PAST)
      __builtin_nontemporal_store(f, (f4*)((float*)p + at));
    else
      *(f4*)((float*)p + at) = f;
  } else if (n > 0) {
#pragma unroll
    for (int e = 0; e < 3; ++e)
      if (e < n) {
        if (bf)
          ((uint16_t*)p)[at + e] = f2bf(v[e]);
        else
          ((float*)p)[at + e] = v[e];
      }
  }
}

template <int CTRL>
__device__ inline float dpp_add(float v) {
  return v + __int_as_float(
                 __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over the workgroup, the same on every thread (rows of 16 lanes by DPP, the
// four rows and the waves in order); `part` is used once.  The barrier is for LDS
// alone, so that it does not wait for loads and stores under way.
template <int THREADS>
__device__ inline float group_sum(float v, float* part) {
  v = dpp_add<0xB1>(v);   // lane ^ 1, lane ^ 2, halves of the row and the row mirrored
  v = dpp_add<0x4E>(v);
  v = dpp_add<0x141>(v);
  v = dpp_add<0x140>(v);
  const float r0 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0));
  const float r1 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16));
  const float r2 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 32));
  const float r3 = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 48));
  v = (r0 + r1) + (r2 + r3);
  if constexpr (THREADS > 64) {
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < THREADS / 64; ++k) v += part[k];
  }
  return v;
}

// NPER runs of four values per thread (4 * NPER * THREADS >= d).  AHEAD: everything
// is loaded before the first sum, for few rows, where weights and gate loaded at
// their use cost a memory latency each (16 rows of 4096: 6.9 us, ahead 3.7).  For
// many rows the registers that this takes cost more than other rows hide (4096
// rows of 8192: 108 us, at their use 82).
template <int THREADS, int NPER, bool AHEAD, bool PAST>
__global__ __launch_bounds__(THREADS) void block_norm_kernel(NormArgs a) {
  __shared__ float part[2][THREADS / 64];
  const int64_t row = (a.row0 + blockIdx.x) * a.d;
  const int64_t grow = (a.row0 + blockIdx.x) * a.gate_stride;
  float x[NPER][4], u[NPER][4], g[NPER][4], post[NPER][4], pre[NPER][4];
  auto load_rest = [&](int i, int c, int n) {
    if (a.post_w) load_row(a.post_w, false, c, n, post[i]);
    if (a.gate) load_row(a.gate, a.g_bf, grow + c, n, g[i]);
    if (a.pre_w) load_row(a.pre_w, false, c, n, pre[i]);
  };
#pragma unroll
  for (int i = 0; i < NPER; ++i) {
    const int c = (threadIdx.x + i * THREADS) * 4, n = a.d - c;
    load_row(a.y, a.y_bf, row + c, n, u[i]);
    load_row(a.x, false, row + c, n, x[i]);
    if constexpr (AHEAD) load_rest(i, c, n);
  }
  if (a.post_w) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < NPER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) ss = fmaf(u[i][e], u[i][e], ss);
    const float inv = 1.0f / sqrtf(group_sum<THREADS>(ss, part[0]) / (float)a.d + a.eps);
#pragma unroll
    for (int i = 0; i < NPER; ++i) {
      const int c = (threadIdx.x + i * THREADS) * 4;
      if constexpr (!AHEAD) load_row(a.post_w, false, c, a.d - c, post[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[i][e] = u[i][e] * inv * post[i][e];
    }
  }
  if (a.gate) {
#pragma unroll
    for (int i = 0; i < NPER; ++i) {
      const int c = (threadIdx.x + i * THREADS) * 4;
      if constexpr (!AHEAD) load_row(a.gate, a.g_bf, grow + c, a.d - c, g[i]);
#pragma unroll
      for (int e = 0; e < 4; ++e) u[i][e] *= g[i][e];
    }
  }
  float ss = 0.0f;
#pragma unroll
  for (int i = 0; i < NPER; ++i) {
    const int c = (threadIdx.x + i * THREADS) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[i][e] = fmaf(a.y_scale, u[i][e], a.x_scale * x[i][e]);
      ss = fmaf(x[i][e], x[i][e], ss);  // zero past the row
    }
    store_row<PAST>(a.x, false, row + c, a.d - c, x[i]);
  }
  if (!a.h) return;
  const float inv = 1.0f / sqrtf(group_sum<THREADS>(ss, part[1]) / (float)a.d + a.eps);
#pragma unroll
  for (int i = 0; i < NPER; ++i) {
    const int c = (threadIdx.x + i * THREADS) * 4;
    if constexpr (!AHEAD)
      if (a.pre_w) load_row(a.pre_w, false, c, a.d - c, pre[i]);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i][e] *= a.pre_w ? inv * pre[i][e] : inv;
    store_row<PAST>(a.h, a.h_bf, row + c, a.d - c, x[i]);
  }
}

template <int THREADS, int NPER, bool AHEAD, bool PAST>
void run_block_norm_n(const NormArgs& a, int T, hipStream_t s) {
  // a grid has fewer than 2^32 threads
  constexpr int kRows = 1 << 21;
  for (NormArgs b = a; b.row0 < T; b.row0 += kRows)
    block_norm_kernel<THREADS, NPER, AHEAD, PAST>
        <<<T - b.row0 < kRows ? T - b.row0 : kRows, THREADS, 0, s>>>(b);
}

// Threads a row, by its runs of four values: one run a thread leaves the shortest
// chain; where rows fill the chip several times over, more runs for wide rows.
// Measured, bf16 with both norms and one gate row, us (threads, runs): 16 rows of
// 4096: (1024, 1) 3.7, (512, 2) 3.9, (256, 4) 5.2; 8192 rows of 4096: 85.5, 82.6
// (4.9 TB/s), 92.2; 16 rows of 8192: (1024, 2) 4.7, (512, 4) 5.6; 4096 rows of
// 8192: 81.5, 99.2; 2048 rows of 16384: (1024, 4) 94, (512, 8) 135.
hipError_t run_block_norm(const NormArgs& a, int T, hipStream_t s) {
  const int n = (a.d + 3) / 4;
  const bool few = T <= 256;                        // one row a CU
  const bool held = (int64_t)T * a.d <= (4 << 20);  // x stays in the L2s (4 MB a XCD)
  if (n <= 64)
    held ? run_block_norm_n<64, 1, true, false>(a, T, s) : run_block_norm_n<64, 1, true, true>(a, T, s);
  else if (n <= 256)
    held ? run_block_norm_n<256, 1, true, false>(a, T, s)
         : run_block_norm_n<256, 1, true, true>(a, T, s);
  else if (n <= 512)
    held ? run_block_norm_n<512, 1, true, false>(a, T, s)
         : run_block_norm_n<512, 1, true, true>(a, T, s);
  else if (n <= 1024)
    few    ? run_block_norm_n<1024, 1, true, false>(a, T, s)
    : held ? run_block_norm_n<512, 2, false, false>(a, T, s)
           : run_block_norm_n<512, 2, false, true>(a, T, s);
  else if (n <= 2048)
    few    ? run_block_norm_n<1024, 2, true, false>(a, T, s)
    : held ? run_block_norm_n<1024, 2, false, false>(a, T, s)
           : run_block_norm_n<1024, 2, false, true>(a, T, s);
  else
    held ? run_block_norm_n<1024, 4, false, false>(a, T, s)
         : run_block_norm_n<1024, 4, false, true>(a, T, s);
  return hipGetLastError();
}

}  // namespace

static_assert(kNormMax <= 4 * 4 * 1024, "a row fits the widest kernel");

hipError_t launch_block_norm(float* x, float x_scale, const void* y, d2moe_dtype yd, float y_scale,
                             const float* post_w, const void* gate, d2moe_dtype gd,
                             int64_t gate_stride, const float* pre_w, int T, int d, float eps,
                             void* h, d2moe_dtype hd, hipStream_t s) {
  if (T == 0) return hipSuccess;
  NormArgs a{};
  a.x = x, a.y = y, a.gate = gate, a.post_w = post_w, a.pre_w = pre_w, a.h = h;
  a.gate_stride = gate_stride, a.x_scale = x_scale, a.y_scale = y_scale, a.eps = eps, a.d = d;
  a.y_bf = yd == D2MOE_BF16, a.g_bf = gd == D2MOE_BF16, a.h_bf = hd == D2MOE_BF16;
  return run_block_norm(a, T, s);
}

}  // namespace d2moe
