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

__device__ inline void store_row(void* p, bool bf, int64_t at, int n, const float (&v)[4]) {
  if (n >= 4) {
    if (bf)
      *(h4*)((uint16_t*)p + at) = h4{f2bf(v[0]), f2bf(v[1]), f2bf(v[2]), f2bf(v[3])};
    else
      *(f4*)((float*)p + at) = f4{v[0], v[1], v[2], v[3]};
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

// NPER runs of four values per thread (4 * NPER * THREADS >= d).  Everything is
// loaded before the first sum: weights and gate loaded where they are used cost a
// memory latency each (16 rows of 4096: 6.9 us).
template <int THREADS, int NPER>
__global__ __launch_bounds__(THREADS) void block_norm_kernel(NormArgs a) {
  __shared__ float part[2][THREADS / 64];
  const int64_t row = (int64_t)blockIdx.x * a.d;
  const int64_t grow = (int64_t)blockIdx.x * a.gate_stride;
  float x[NPER][4], u[NPER][4], g[NPER][4], post[NPER][4], pre[NPER][4];
#pragma unroll
  for (int i = 0; i < NPER; ++i) {
    const int c = (threadIdx.x + i * THREADS) * 4, n = a.d - c;
    load_row(a.y, a.y_bf, row + c, n, u[i]);
    load_row(a.x, false, row + c, n, x[i]);
    if (a.post_w) load_row(a.post_w, false, c, n, post[i]);
    if (a.gate) load_row(a.gate, a.g_bf, grow + c, n, g[i]);
    if (a.pre_w) load_row(a.pre_w, false, c, n, pre[i]);
  }
  if (a.post_w) {
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < NPER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) ss = fmaf(u[i][e], u[i][e], ss);
    const float inv = 1.0f / sqrtf(group_sum<THREADS>(ss, part[0]) / (float)a.d + a.eps);
#pragma unroll
    for (int i = 0; i < NPER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) u[i][e] = u[i][e] * inv * post[i][e];
  }
  if (a.gate) {
#pragma unroll
    for (int i = 0; i < NPER; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) u[i][e] *= g[i][e];
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
    store_row(a.x, false, row + c, a.d - c, x[i]);
  }
  if (!a.h) return;
  const float inv = 1.0f / sqrtf(group_sum<THREADS>(ss, part[1]) / (float)a.d + a.eps);
#pragma unroll
  for (int i = 0; i < NPER; ++i) {
    const int c = (threadIdx.x + i * THREADS) * 4;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[i][e] *= a.pre_w ? inv * pre[i][e] : inv;
    store_row(a.h, a.h_bf, row + c, a.d - c, x[i]);
  }
}

// Threads a row, by its runs of four values.  One run a thread leaves the shortest
// chain; where rows fill the chip several times over, workgroups of 512 overlap
// better.  Measured, bf16 with both norms and a gate for all rows, us (threads,
// runs): 16 rows of 4096: (1024, 1) 3.73, (512, 2) 3.89, (256, 4) 5.16; 8192 rows of
// 4096: 70.7, 62.4, 69.4; 16 rows of 8192: (1024, 2) 4.74, (512, 4) 5.61; 4096 rows
// of 8192: 77.0, 73.3; 8192 rows of 2048: (512, 1) 33.1 (6.1 TB/s), (1024, 1) 52.6.
hipError_t run_block_norm(const NormArgs& a, int T, hipStream_t s) {
  const int n = (a.d + 3) / 4;
  const bool few = T <= 256;  // one row a CU
  if (n <= 64)
    block_norm_kernel<64, 1><<<T, 64, 0, s>>>(a);
  else if (n <= 256)
    block_norm_kernel<256, 1><<<T, 256, 0, s>>>(a);
  else if (n <= 512)
    block_norm_kernel<512, 1><<<T, 512, 0, s>>>(a);
  else if (n <= 1024 && few)
    block_norm_kernel<1024, 1><<<T, 1024, 0, s>>>(a);
  else if (n <= 1024)
    block_norm_kernel<512, 2><<<T, 512, 0, s>>>(a);
  else if (n <= 2048 && few)
    block_norm_kernel<1024, 2><<<T, 1024, 0, s>>>(a);
  else if (n <= 2048)
    block_norm_kernel<512, 4><<<T, 512, 0, s>>>(a);
  else
    block_norm_kernel<512, 8><<<T, 512, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace

static_assert(kNormMax <= 4 * 8 * 512, "a row fits the widest kernel");

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
