// Linear layers with 4-bit weights and group scales,
//   y[t][r] = bias[r] + sum_g s[r][g] (sum_{c in g} n[r][c] x[t][c] - z[r][g] sum_{c in g} x[t][c])
// on v_mfma_f32_16x16x32_bf16: lane 16 q + i holds row i, columns 8 q .. 8 q + 7
// of either operand, and rows 4 q .. 4 q + 3 of column i of the result.
//
// A code n becomes the bf16 number 16 + n by placing its four bits below the
// leading one of 16 (0x4180): one shift and one and-or for two codes, exact.
// The product with the 16 + z that has to be taken off again uses the sum of
// x over the group, which a second MFMA with a matrix of ones leaves in the
// same lanes as the first one's results.  16 rather than a larger power of two
// keeps the two parts near the result's size (31 / 15 at most in the weights),
// so the difference costs about one bit of binary32.
//
// bf16 activations are used as they are; binary32 ones as the sum of three
// bf16 pieces of 8 bits each, which is exact.
#include "decoder.h"

namespace d2moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

struct LinArgs {
  const void* x;
  const uint32_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const float* bias;
  void* y;
  int T, rows, cols, KB;
  bool y_bf;
};

// The empty asm reads the operands after the result exists, so that the result
// is never given some of their registers (an MFMA may read its sources while it
// writes).
__device__ inline f4 mma(u4 a, u4 b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

// The eight codes of a word as 16 + n in bf16 (pair p: codes 2 p, 2 p + 1).
__device__ inline u4 decode(uint32_t w) {
  constexpr uint32_t kMask = 0x00780078u, kOne = 0x41804180u;
  return u4{((w << 3) & kMask) | kOne, ((w >> 1) & kMask) | kOne, ((w >> 5) & kMask) | kOne,
            ((w >> 9) & kMask) | kOne};
}

// The operand(s) of eight activations: NP = 1 for bf16, 3 pieces for binary32,
// smallest first.  A piece is the value cut to its upper 16 bits, what is left
// goes to the next; nothing is left of an infinity or NaN.
template <int NP>
struct XFrag {
  u4 p[NP];
};
__device__ inline XFrag<1> load_x(const uint16_t* x) { return {*(const u4*)x}; }
__device__ inline XFrag<3> load_x(const float* x) {
  const f4 a = *(const f4*)x, b = *(const f4*)(x + 4);
  XFrag<3> f;
  uint32_t h[3][8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float v = e < 4 ? a[e & 3] : b[e & 3];
    const bool finite = (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u;
#pragma unroll
    for (int k = 2; k >= 0; --k) {
      h[k][e] = __float_as_uint(v) & 0xffff0000u;
      v -= __uint_as_float(h[k][e]);
      v = finite ? v : 0.0f;
    }
  }
#pragma unroll
  for (int k = 0; k < 3; ++k)
#pragma unroll
    for (int d = 0; d < 4; ++d) f.p[k][d] = h[k][2 * d + 1] | h[k][2 * d] >> 16;
  return f;
}

// A workgroup computes 16 rows by 16 NT tokens; its WAVES waves take column
// blocks in turn and add up through LDS.  GB groups per block of 128 columns.
template <typename TX, int NT, int GB, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void linear_kernel(LinArgs a) {
  constexpr int NP = sizeof(TX) == 2 ? 1 : 3;
  __shared__ f4 part[WAVES][NT][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = lane >> 4;
  const int rb = blockIdx.x, t0 = blockIdx.y * 16 * NT;
  const TX* xr[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    // tokens past the end repeat the last one; their results are not written
    const int t = t0 + 16 * n + (lane & 15);
    xr[n] = (const TX*)a.x + (int64_t)(t < a.T ? t : a.T - 1) * a.cols + 8 * q;
  }
  const u4 ones = {0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
  f4 y[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) y[n] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int kb = wave; kb < a.KB; kb += WAVES) {
    const size_t blk = (size_t)rb * a.KB + kb;
    const u4 w = *(const u4*)(a.codes + (blk * 64 + lane) * 4);
    const uint16_t* sp = a.scales + blk * GB * kLinRows + 4 * q;
    const uint8_t* zp = a.zeros + blk * GB * kLinRows + 4 * q;
    const int c0 = kb * kLinCols;
#pragma unroll
    for (int g = 0; g < GB; ++g) {
      const uint2 sw = *(const uint2*)(sp + g * kLinRows);
      const uint32_t zw = *(const uint32_t*)(zp + g * kLinRows);
      f4 acc[NT], xs[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[n] = xs[n] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int jj = 0; jj < 4 / GB; ++jj) {
        const int j = g * (4 / GB) + jj;
        // past the last column (cols is a multiple of 32) the scale is zero
        // and any columns of the same token do
        const int c = GB > 1 && c0 + 32 * j >= a.cols ? c0 : c0 + 32 * j;
        const u4 wa = decode(w[j]);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const XFrag<NP> xf = load_x(xr[n] + c);
#pragma unroll
          for (int k = 0; k < NP; ++k) {
            acc[n] = mma(wa, xf.p[k], acc[n]);
            xs[n] = mma(ones, xf.p[k], xs[n]);
          }
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float s = h2f((uint16_t)((i < 2 ? sw.x : sw.y) >> (16 * (i & 1))));
        const float z = 16.0f + (float)((zw >> (8 * i)) & 255u);
#pragma unroll
        for (int n = 0; n < NT; ++n) y[n][i] = fmaf(s, fmaf(-z, xs[n][i], acc[n][i]), y[n][i]);
      }
    }
  }
#pragma unroll
  for (int n = 0; n < NT; ++n) part[wave][n][lane] = y[n];
  __syncthreads();
  // result r of token t lies in lane 16 (r / 4) + t % 16 of tile t / 16, row r % 4
  for (int o = threadIdx.x; o < 256 * NT; o += 64 * WAVES) {
    const int r = o & 15, t = o >> 4, row = rb * kLinRows + r;
    if (row >= a.rows || t0 + t >= a.T) continue;
    float sum = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += part[w][t >> 4][(r >> 2) * 16 + (t & 15)][r & 3];
    if (a.bias) sum += a.bias[row];
    const int64_t at = (int64_t)(t0 + t) * a.rows + row;
    if (a.y_bf)
      ((uint16_t*)a.y)[at] = f2bf(sum);
    else
      ((float*)a.y)[at] = sum;
  }
}

template <typename TX, int NT, int WAVES>
hipError_t run_linear_g(const LinArgs& a, int group, hipStream_t s) {
  const dim3 grid((a.rows - 1) / kLinRows + 1, (a.T - 1) / (16 * NT) + 1);
  if (group == 128)
    linear_kernel<TX, NT, 1, WAVES><<<grid, 64 * WAVES, 0, s>>>(a);
  else if (group == 64)
    linear_kernel<TX, NT, 2, WAVES><<<grid, 64 * WAVES, 0, s>>>(a);
  else
    linear_kernel<TX, NT, 4, WAVES><<<grid, 64 * WAVES, 0, s>>>(a);
  return hipGetLastError();
}

template <typename TX>
hipError_t run_linear(const LinArgs& a, int group, hipStream_t s) {
  if (a.T <= 16) return run_linear_g<TX, 1, 8>(a, group, s);
  if (a.T <= 32) return run_linear_g<TX, 2, 8>(a, group, s);
  return run_linear_g<TX, 4, 8>(a, group, s);
}

}  // namespace

hipError_t launch_linear(const void* x, d2moe_dtype xd, int T, const d2moe_linear* w,
                         const float* bias, void* y, d2moe_dtype yd, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const LinArgs a{x, w->codes, w->scales, w->zeros, bias, y, T, w->rows, w->cols,
                  lin_col_blocks(w), yd == D2MOE_BF16};
  return xd == D2MOE_BF16 ? run_linear<uint16_t>(a, w->group, s)
                          : run_linear<float>(a, w->group, s);
}

}  // namespace d2moe
