// 4-bit linear layers: quantize + pack (the base level of Eq. 2 at four bits)
// and the packing of given codes.
//
// The codes are integers decided by binary32 arithmetic, so this file is
// compiled without FMA contraction, like pack.hip.
#pragma clang fp contract(off)

#include "decoder.h"

namespace d2moe {
namespace {

constexpr int kPackWaves = 4;  // column blocks (one per wave) of a workgroup

struct LinOut {
  int rows, cols, group, KB;
  uint32_t* codes;
  uint16_t* scales;
  uint8_t* zeros;
};

// Where code e of a word lies: even codes in the low half, odd ones in the
// high half, so that one shift brings two neighbours to the same place of
// their halves.
__device__ inline int code_bit(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// One wave packs one block: lane l holds the 32 weights of row 16 rb + l % 16
// at columns 32 j + 8 (l / 16) + e, the ones of its four words.  A group of 32,
// 64 or 128 columns is 1, 2 or 4 values of j over the four lanes of a row; its
// extremes come by two exchanges.  Setup work, bound by reading W (4 bytes in,
// half a byte out).
__global__ __launch_bounds__(64 * kPackWaves) void linear_pack_kernel(const float* __restrict__ W,
                                                                      LinOut o) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int rb = blockIdx.x, kb = blockIdx.y * kPackWaves + (threadIdx.x >> 6);
  if (kb >= o.KB) return;
  const int row = rb * kLinRows + r;
  const size_t blk = (size_t)rb * o.KB + kb;
  const int per = o.group / 32, gb = 4 / per;  // words per group, groups per block
  float w[4][8];
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int c = kb * kLinCols + 32 * j + 8 * q + e;
      w[j][e] = row < o.rows && c < o.cols ? W[(size_t)row * o.cols + c] : 0.0f;
    }
  float lo[4], hi[4];  // of the group that word j belongs to
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float mn = 0.0f, mx = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      mn = w[j][e] < mn ? w[j][e] : mn;
      mx = w[j][e] > mx ? w[j][e] : mx;
    }
    for (int off = 16; off < 64; off <<= 1) {
      mn = fminf(mn, __shfl_xor(mn, off, 64));
      mx = fmaxf(mx, __shfl_xor(mx, off, 64));
    }
    lo[j] = mn;
    hi[j] = mx;
  }
  if (per >= 2) {
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      lo[j] = lo[j + 1] = fminf(lo[j], lo[j + 1]);
      hi[j] = hi[j + 1] = fmaxf(hi[j], hi[j + 1]);
    }
  }
  if (per == 4) {
    lo[0] = lo[1] = lo[2] = lo[3] = fminf(lo[0], lo[2]);
    hi[0] = hi[1] = hi[2] = hi[3] = fmaxf(hi[0], hi[2]);
  }
  uint32_t word[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const bool inside = row < o.rows && kb * kLinCols + 32 * j < o.cols;
    uint16_t s_h = f2h((hi[j] - lo[j]) / 15.0f);
    float s = h2f(s_h);
    if (!(s > 0.0f) || __builtin_isinf(s)) {
      s_h = 0x3c00u;
      s = 1.0f;
    }
    float z = rintf(-lo[j] / s);
    z = z < 0.0f ? 0.0f : z;
    z = z > 15.0f ? 15.0f : z;
    word[j] = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      // clamped to [0, 15]; NaN gives 0
      const float n = __builtin_amdgcn_fmed3f(rintf(w[j][e] / s + z), 0.0f, 15.0f);
      word[j] |= (uint32_t)(int)n << code_bit(e);
    }
    if (!inside) {
      word[j] = 0;
      s_h = 0;
      z = 0.0f;
    }
    if (q == 0 && j % per == 0) {
      const size_t at = (blk * gb + j / per) * kLinRows + r;
      o.scales[at] = s_h;
      o.zeros[at] = (uint8_t)(16 + (int)z);
    }
  }
  *(uint4*)(o.codes + (blk * 64 + lane) * 4) = make_uint4(word[0], word[1], word[2], word[3]);
}

// The same walk over given codes, scales and zero points.
__global__ __launch_bounds__(64 * kPackWaves) void linear_pack_codes_kernel(
    const uint8_t* __restrict__ codes, const uint16_t* __restrict__ scales,
    const uint8_t* __restrict__ zeros, LinOut o) {
  const int lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
  const int rb = blockIdx.x, kb = blockIdx.y * kPackWaves + (threadIdx.x >> 6);
  if (kb >= o.KB) return;
  const int row = rb * kLinRows + r;
  const size_t blk = (size_t)rb * o.KB + kb;
  const int per = o.group / 32, gb = 4 / per;
  uint32_t word[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c = kb * kLinCols + 32 * j;
    const bool inside = row < o.rows && c < o.cols;
    word[j] = 0;
    if (inside)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        word[j] |= (uint32_t)(codes[(size_t)row * o.cols + c + 8 * q + e] & 15) << code_bit(e);
    if (q == 0 && j % per == 0) {
      const size_t at = (blk * gb + j / per) * kLinRows + r;
      const size_t from = (size_t)row * (o.cols / o.group) + c / o.group;
      o.scales[at] = inside ? scales[from] : (uint16_t)0;
      o.zeros[at] = (uint8_t)(16 + (!inside ? 0 : zeros ? zeros[from] & 15 : 8));
    }
  }
  *(uint4*)(o.codes + (blk * 64 + lane) * 4) = make_uint4(word[0], word[1], word[2], word[3]);
}

LinOut out_of(const d2moe_linear* w) {
  return LinOut{w->rows, w->cols, w->group, lin_col_blocks(w), w->codes, w->scales, w->zeros};
}

dim3 pack_grid(const d2moe_linear* w) {
  return dim3(lin_row_blocks(w), (lin_col_blocks(w) + kPackWaves - 1) / kPackWaves);
}

}  // namespace

hipError_t launch_linear_pack(const float* W, const d2moe_linear* out, hipStream_t s) {
  linear_pack_kernel<<<pack_grid(out), 64 * kPackWaves, 0, s>>>(W, out_of(out));
  return hipGetLastError();
}

hipError_t launch_linear_pack_codes(const uint8_t* codes, const uint16_t* scales,
                                    const uint8_t* zeros, const d2moe_linear* out, hipStream_t s) {
  linear_pack_codes_kernel<<<pack_grid(out), 64 * kPackWaves, 0, s>>>(codes, scales, zeros,
                                                                     out_of(out));
  return hipGetLastError();
}

}  // namespace d2moe
