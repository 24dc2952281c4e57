// Linear layers with 4-bit weights and group scales,
//   y[t][r] = bias[r] + sum_g s[r][g] (sum_{c in g} n[r][c] x[t][c] - z[r][g] sum_{c in g} x[t][c])
// on v_mfma_f32_16x16x32_bf16: lane 16 q + i holds row i, columns 8 q .. 8 q + 7
// of either operand, and rows 4 q .. 4 q + 3 of column i of the result.
//
// A code n becomes the bf16 number 16 + n by placing its four bits below the
// leading one of 16 (0x4180): one shift and one and-or for two codes, exact.
// 16 + z times the sum of x over the group is taken off again.  16 rather than a
// larger power of two keeps the two parts near the result's size (31 / 15 at
// most in the weights), so the difference costs about one bit of binary32.
//
// bf16 activations are used as they are; binary32 ones as the sum of three
// bf16 pieces of 8 bits each, which is exact.
#include <type_traits>

#include "decoder.h"

namespace d2moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));
// four results of a token, whose row starts at any element
typedef float row4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t row4h __attribute__((ext_vector_type(4), aligned(2)));

struct LinArgs {
  const void* x;
  const uint32_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const float* bias;
  void* y;
  int T, rows, cols, RB, KB;
  bool y_bf;
};

// The empty asm reads the operands after the result exists, so that the result
// is never given some of their registers (an MFMA may read its sources while it
// writes).
__device__ inline f4 mma(u4 a, u4 b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));
  return d;
}

// The eight codes of a word as 16 + n in bf16 (pair p: codes 2 p, 2 p + 1), a
// shift and an and-or each.  The instruction takes one constant from outside
// the vector registers, so the mask is held in one.
__device__ inline uint32_t code_mask() {
  uint32_t m = 0x00780078u;
  asm("" : "+v"(m));
  return m;
}
__device__ inline u4 decode(uint32_t w, uint32_t mask) {
  constexpr uint32_t kOne = 0x41804180u;
  return u4{((w << 3) & mask) | kOne, ((w >> 1) & mask) | kOne, ((w >> 5) & mask) | kOne,
            ((w >> 9) & mask) | kOne};
}

// Eight activations as loaded; the operand(s) they become (NP = 1 for bf16, 3
// pieces for binary32, smallest first) and their sums.  A piece is the value cut
// to its upper 16 bits, what is left goes to the next (an infinity leaves NaN).
template <typename TX>
struct XRaw;
template <>
struct XRaw<uint16_t> {
  static constexpr int NP = 1;
  u4 v;
  __device__ void load(const uint16_t* x) { v = *(const u4*)x; }
  __device__ void pieces(u4 (&p)[1]) const { p[0] = v; }
  __device__ void sum(float (&s)[1]) const {
    const b2 one = {(__bf16)1.0f, (__bf16)1.0f};
    s[0] = 0.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
      s[0] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, (uint32_t)v[d]), one, s[0],
                                             false);
  }
};
template <>
struct XRaw<float> {
  static constexpr int NP = 3;
  f4 v[2];
  __device__ void load(const float* x) {
    v[0] = *(const f4*)x;
    v[1] = *(const f4*)(x + 4);
  }
  __device__ void pieces(u4 (&p)[3]) const {
    uint32_t h[3][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float f = v[e >> 2][e & 3];
#pragma unroll
      for (int k = 2; k >= 0; --k) {
        h[k][e] = __float_as_uint(f);
        f -= __uint_as_float(h[k][e] & 0xffff0000u);
      }
    }
#pragma unroll
    for (int k = 0; k < 3; ++k)
#pragma unroll
      for (int d = 0; d < 4; ++d)
        p[k][d] = __builtin_amdgcn_perm(h[k][2 * d + 1], h[k][2 * d], 0x07060302u);
  }
  __device__ void sum(float (&s)[2]) const {  // of the first pieces and of what is left
    s[0] = s[1] = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float f = v[e >> 2][e & 3];
      const float first = __uint_as_float(__float_as_uint(f) & 0xffff0000u);
      s[0] += first;
      s[1] += f - first;
    }
  }
};

template <int CTRL>
__device__ inline float dpp_add(float v) {
  return v + __int_as_float(
                 __builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// A barrier for LDS alone: a full one would also wait for the loads under way.
__device__ inline void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ inline void put(const LinArgs& a, int64_t at, float v) {
  if (a.y_bf)
    ((uint16_t*)a.y)[at] = f2bf(v);
  else
    ((float*)a.y)[at] = v;
}

// What a lane needs of one column block for RT row tiles, beside x.
template <int RT, int GB>
struct WFrag {
  u4 w[RT];
  uint2 s[RT][GB];     // four binary16 scales, rows 4 q .. 4 q + 3
  uint32_t z[RT][GB];  // 16 + their zero points
};
template <int RT, int GB>
__device__ inline void load_w(WFrag<RT, GB>& f, const LinArgs& a, int rb0, int kb, int lane) {
  const uint32_t q = lane >> 4;
#pragma unroll
  for (int r = 0; r < RT; ++r) {
    // row tiles past the end repeat the last one (their results are not
    // written), and so do column blocks (their scales are taken as zero)
    const int rb = rb0 + r < a.RB ? rb0 + r : a.RB - 1;
    const size_t blk = (size_t)rb * a.KB + (kb < a.KB ? kb : a.KB - 1);
    f.w[r] = *(const u4*)((const char*)a.codes + blk * 1024 + 16u * lane);
    const char* sp = (const char*)a.scales + blk * (GB * kLinRows * 2);
    const char* zp = (const char*)a.zeros + blk * (GB * kLinRows);
#pragma unroll
    for (int g = 0; g < GB; ++g) {
      f.s[r][g] = *(const uint2*)(sp + (8u * q + g * kLinRows * 2));
      f.z[r][g] = *(const uint32_t*)(zp + (4u * q + g * kLinRows));
    }
  }
}

// A workgroup computes 16 RT R rows by 16 NT tokens: R waves side by side in the
// rows times S that take column blocks in turn and add up through LDS.  GB
// groups per block of 128 columns.
//
// The activations of a column block go through LDS, for the R waves that share
// them and because rows of them are whole cache lines while an operand is 16
// pieces of 64 bytes, which the L1 takes twice as long for.  The 16-byte piece of
// token t, columns 8 c .. 8 c + 7 of the block, lies where lane (c % 4, t % 16 ^ c)
// of operand c / 4 reads it: 16 neighbouring lanes meet 16 different bank groups
// writing (one token) and reading (one c).  The group sums of x are taken on the
// way.
//
// Weights and activations are loaded two steps before their use.
template <typename TX, int NT, int NU, int RT, int R, int S, int GB>
__global__ __launch_bounds__(64 * R * S) void linear_kernel(LinArgs a) {
  constexpr int NP = XRaw<TX>::NP, kUnits = (NU + R - 1) / R;
  // The first pieces of binary32 activations are summed apart from the rest, here and
  // in the sums of x: they have 8 bits, their products 13, so both sums are nearly
  // exact, and what the 16 + z cancels of them is not rounded at the size of the
  // uncancelled sums (one group of 128 columns: errors of 3e-8 of the result, with
  // one sum of x 1e-6; 16 x 4096 x 4096 takes 11.2 us for it, 10.9 with one).
  constexpr int NA = NP == 1 ? 1 : 2;
  struct Stage {
    u4 x[2][S][NP][NT * 4 * 64];
    float sum[2][S][NA][GB][NT * 16];
  };
  union Lds {
    Stage st;
    f4 part[S][R * RT][NT][64];
  };
  __shared__ Lds lds;
  const int lane = threadIdx.x & 63, q = lane >> 4, col = lane & 15;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // addresses stay scalar
  const int rw = wave % R, sk = wave / R;
  const int rb0 = (blockIdx.x * R + rw) * RT, t0 = blockIdx.y * 16 * NT;
  const int steps = (a.KB + S - 1) / S;

  // NU units of 4 tokens by 128 columns (fewer than 4 NT where there are no more
  // tokens); a lane has 8 columns of one token.  Tokens past the last repeat it
  // (their results are not written), and so do columns (their groups are left out)
  // and blocks (their scales are taken as zero): every load is made, so that a wait can
  // count on those behind the one it is for.
  uint32_t xrow[kUnits];
#pragma unroll
  for (int i = 0; i < kUnits; ++i) {
    const int t = 4 * (rw + R * i) + q;
    xrow[i] = (uint32_t)(t < a.T - t0 ? t : a.T - t0 - 1) * a.cols;
  }
  auto load_x = [&](XRaw<TX> (&x)[kUnits], int kb) {
    const int c0 = (kb < a.KB ? kb : a.KB - 1) * kLinCols;
    const char* xk = (const char*)a.x + ((int64_t)t0 * a.cols + c0) * sizeof(TX);
    int c = 8 * col;
    if constexpr (GB > 1) c = c < a.cols - c0 ? c : a.cols - c0 - 8;
#pragma unroll
    for (int i = 0; i < kUnits; ++i) x[i].load((const TX*)(xk + (xrow[i] + c) * (uint32_t)sizeof(TX)));
  };
  auto store_x = [&](const XRaw<TX> (&x)[kUnits], int buf) {
#pragma unroll
    for (int i = 0; i < kUnits; ++i) {
      const int unit = rw + R * i;
      if (NU % R != 0 && unit >= NU) break;
      const int t = 4 * unit + q;
      u4 p[NP];
      x[i].pieces(p);
#pragma unroll
      for (int k = 0; k < NP; ++k)
        lds.st.x[buf][sk][k][((t >> 4) * 4 + (col >> 2)) * 64 + (col & 3) * 16 +
                             ((t & 15) ^ col)] = p[k];
      float s[NA];
      x[i].sum(s);
#pragma unroll
      for (int h = 0; h < NA; ++h) {
        s[h] = dpp_add<0xB1>(s[h]);  // quads: lane ^ 1, lane ^ 2
        s[h] = dpp_add<0x4E>(s[h]);
        if constexpr (GB <= 2) s[h] = dpp_add<0x141>(s[h]);  // halves of a row of 16, mirrored
        if constexpr (GB == 1) s[h] = dpp_add<0x140>(s[h]);  // the row, mirrored
      }
      if (col % (16 / GB) == 0) {
#pragma unroll
        for (int h = 0; h < NA; ++h) lds.st.sum[buf][sk][h][col / (16 / GB)][t] = s[h];
      }
    }
  };
  // a step's activations are shared by R waves, or stay within one
  auto hand_over = [&] {
    if constexpr (R > 1) {
      lds_barrier();
    } else {
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
  };

  const uint32_t mask = code_mask();
  const f4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
  float y[RT][NT][4];
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) y[r][n][i] = 0.0f;
  // Step `it` with its weights; x holds the activations of the next step.  Both
  // are loaded again, for two steps on, as soon as they have been used.
  auto step = [&](int it, auto parity, WFrag<RT, GB>& w, XRaw<TX> (&x)[kUnits]) {
    constexpr int buf = decltype(parity)::value;
    const bool live = it * S + sk < a.KB;  // a block past the last one adds nothing
    // operands of the activations, read one word ahead of their products
    u4 xp[2][NT][NP];
    auto read_x = [&](int j) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int k = 0; k < NP; ++k)
          xp[j & 1][n][k] = lds.st.x[buf][sk][k][(n * 4 + j) * 64 + q * 16 + (col ^ (4 * j + q))];
    };
    read_x(0);
    store_x(x, buf ^ 1);  // under the first operands' way from LDS
    load_x(x, (it + 3) * S + sk);
#pragma unroll
    for (int g = 0; g < GB; ++g) {
      f4 acc[RT][NT][NA];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < NA; ++h)
#pragma unroll
          for (int r = 0; r < RT; ++r) acc[r][n][h] = zero;
      float xs[NT][NA];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int h = 0; h < NA; ++h) xs[n][h] = lds.st.sum[buf][sk][h][g][16 * n + col];
#pragma unroll
      for (int jj = 0; jj < 4 / GB; ++jj) {
        const int j = g * (4 / GB) + jj;
        if (j < 3) read_x(j + 1);
        __builtin_amdgcn_sched_barrier(0);
        u4 wa[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r) wa[r] = decode(w.w[r][j], mask);
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int k = 0; k < NP; ++k) {
            const int h = k == NP - 1 ? 0 : 1;
#pragma unroll
            for (int r = 0; r < RT; ++r) acc[r][n][h] = mma(wa[r], xp[j & 1][n][k], acc[r][n][h]);
          }
      }
      // a group past the last column: its sums repeat other columns and may overflow
      // where no group does, so that a scale of zero would not take them out
      if (GB > 1 && (it * S + sk) * kLinCols + g * (kLinCols / GB) >= a.cols) continue;
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        const uint2 sc = live ? w.s[r][g] : make_uint2(0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float s = h2f((uint16_t)((i < 2 ? sc.x : sc.y) >> (16 * (i & 1))));
          const float z = (float)((w.z[r][g] >> (8 * i)) & 255u);  // 16 + zero point
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float v = fmaf(-z, xs[n][0], acc[r][n][0][i]);
            if constexpr (NA == 2) v += fmaf(-z, xs[n][1], acc[r][n][1][i]);
            y[r][n][i] = fmaf(s, v, y[r][n][i]);
          }
        }
      }
    }
    load_w(w, a, rb0, (it + 2) * S + sk, lane);
    hand_over();
  };
  WFrag<RT, GB> w0, w1;
  XRaw<TX> x0[kUnits], x1[kUnits];
  load_x(x0, sk);
  load_w(w0, a, rb0, sk, lane);
  load_x(x1, S + sk);
  load_w(w1, a, rb0, S + sk, lane);
  store_x(x0, 0);
  load_x(x0, 2 * S + sk);
  hand_over();
  for (int it = 0; it < steps; it += 2) {
    step(it, std::integral_constant<int, 0>{}, w0, x1);
    if (it + 1 == steps) break;
    step(it + 1, std::integral_constant<int, 1>{}, w1, x0);
  }
  lds_barrier();  // the buffers become the waves' results
  // A lane's four rows (16 r + 4 q .. + 3 of token 16 n + col) stay together; 8
  // threads that take the quads of one token after the other meet 8 different bank
  // groups.
  auto place = [](int tile, int quad, int t) { return quad * 16 + (t ^ (quad | (tile & 1) << 2)); };
#pragma unroll
  for (int r = 0; r < RT; ++r)
#pragma unroll
    for (int n = 0; n < NT; ++n)
      lds.part[sk][rw * RT + r][n][place(rw * RT + r, q, col)] =
          f4{y[r][n][0], y[r][n][1], y[r][n][2], y[r][n][3]};
  lds_barrier();
  constexpr int kQuads = 4 * R * RT;
  if constexpr (NT * RT >= S) {
    // a quad a thread, where that leaves no thread idle (32000 x 4096 at 64 tokens: 31.1
    // us with a value a thread, 29.9 so; one token of 4096 x 4096: 4.2 and 4.5)
    for (int o = threadIdx.x; o < kQuads * 16 * NT; o += 64 * R * S) {
      const int i = o % kQuads, t = o / kQuads, row = (blockIdx.x * kQuads + i) * 4;
      if (row >= a.rows || t0 + t >= a.T) continue;
      f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < S; ++w) sum += lds.part[w][i >> 2][t >> 4][place(i >> 2, i & 3, t & 15)];
      const int64_t to = (int64_t)(t0 + t) * a.rows + row;
      if (row + 4 <= a.rows) {
        if (a.bias) sum += *(const row4*)(a.bias + row);
        if (a.y_bf)
          *(row4h*)((uint16_t*)a.y + to) =
              row4h{f2bf(sum[0]), f2bf(sum[1]), f2bf(sum[2]), f2bf(sum[3])};
        else
          *(row4*)((float*)a.y + to) = sum;
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (row + e < a.rows) put(a, to + e, sum[e] + (a.bias ? a.bias[row + e] : 0.0f));
      }
    }
  } else {
    for (int o = threadIdx.x; o < kQuads * 64 * NT; o += 64 * R * S) {
      const int i = o % (4 * kQuads), t = o / (4 * kQuads), row = blockIdx.x * 4 * kQuads + i;
      if (row >= a.rows || t0 + t >= a.T) continue;
      float sum = 0.0f;
#pragma unroll
      for (int w = 0; w < S; ++w)
        sum += lds.part[w][i >> 4][t >> 4][place(i >> 4, i >> 2 & 3, t & 15)][i & 3];
      put(a, (int64_t)(t0 + t) * a.rows + row, sum + (a.bias ? a.bias[row] : 0.0f));
    }
  }
}

template <typename TX, int NT, int NU, int RT, int R, int S, int GB>
hipError_t run_linear_g(const LinArgs& a, hipStream_t s) {
  const dim3 grid((a.RB - 1) / (RT * R) + 1, (a.T - 1) / (16 * NT) + 1);
  linear_kernel<TX, NT, NU, RT, R, S, GB><<<grid, 64 * R * S, 0, s>>>(a);
  return hipGetLastError();
}

// The division of the work.  Workgroups of 128 rows by 64 or 32 tokens reuse most,
// and are taken where three quarters of the CUs get one.  Otherwise it goes by
// the number of 16 x 16 tiles of the result: up to one per CU, a workgroup takes
// one tile and its waves divide the columns; with more, 2, 4 and 8 row tiles share
// the activations (whose reading from L2 bounds the kernel otherwise) while one
// round of workgroups fills the chip.  Measured, bf16, 4096 columns, group 128, us:
//   R, S of 16-token workgroups         1, 8   2, 4   4, 4   8, 2
//   4096 rows x 16 (256 tiles)           6.0    6.8    8.3   12.0
//   6144 rows x 16 (384 tiles)           8.7    7.0    8.4   12.0
//   4096 rows x 64 (1024 tiles)         14.3    9.8    8.5   12.0
//   6144 rows x 64 (1536 tiles)         19.8   12.6   15.1   12.1
//   32000 rows x 16                     29.1   19.2   17.5   16.8
//   tokens of a workgroup of 128 rows      16     32     64
//   6144 rows x 64 (192, 96, 48 of them) 12.1   15.9   24.2
//   16384 rows x 64 (512, 256, 128)      24.2   18.1   25.5
//   32000 rows x 64 (1000, 500, 250)     50.7   34.4   26.7
// What bounds the last (2.6 TB/s, 0.63 PFLOP/s) is issue more than any unit: vector
// instructions take 53 % of the issue slots, the matrix units are busy for 28 % of the
// cycles, and of the waves, two a SIMD, 28 % wait and 32 % could not issue.  Some 8 of
// the 27 us are the launch, the first loads and the results, and of the rest decoding,
// scales, sums of x and products each cost what leaving them out saves, 1 to 4 us.
// Binary32 activations take three times the LDS and products.
constexpr int kCus = 256;

template <int NU, int GB>
hipError_t run_linear_16(const LinArgs& a, int64_t tiles, hipStream_t s) {
  if (tiles <= kCus) {
    // long rows at one to four tokens: 16 waves keep more loads under way (14336
    // columns 9.1 us, with 8 waves 10.3; 4096 columns 4.5 and 4.2)
    if constexpr (NU == 1)
      if (a.KB > 48) return run_linear_g<uint16_t, 1, NU, 1, 1, 16, GB>(a, s);
    return run_linear_g<uint16_t, 1, NU, 1, 1, 8, GB>(a, s);
  }
  if (tiles <= 2 * kCus) return run_linear_g<uint16_t, 1, NU, 1, 2, 4, GB>(a, s);
  if (tiles <= 4 * kCus) return run_linear_g<uint16_t, 1, NU, 1, 4, 4, GB>(a, s);
  return run_linear_g<uint16_t, 1, NU, 1, 8, 2, GB>(a, s);
}
template <int NU, int GB>
hipError_t run_linear_32(const LinArgs& a, int64_t tiles, hipStream_t s) {
  if constexpr (NU == 1)
    if (tiles <= kCus) return run_linear_g<float, 1, NU, 1, 1, 6, GB>(a, s);
  // groups of 32 need more registers than 16 waves have
  if (tiles <= 2 * kCus || GB == 4) return run_linear_g<float, 1, NU, 1, 2, 4, GB>(a, s);
  if constexpr (GB < 4) return run_linear_g<float, 1, NU, 1, 4, 4, GB>(a, s);
}

// Workgroups of 128 rows, or of 256, which take 1.63 times as long and are taken
// where that saves rounds of workgroups (one a CU): 6144 x 4096 at 256 tokens (192 or
// 96 workgroups) 24.8 us and 39.4, 32000 x 4096 at 128 (500 or 250) 51.0 and 44.9; fp32,
// 96 tokens (750 or 375) 93 and 101, 128 (1000 or 500) 124 and 106.
template <typename TX, int NT, int GB>
hipError_t run_linear_wide(const LinArgs& a, hipStream_t s) {
  const int64_t blocks = (a.T - 1) / (16 * NT) + 1;
  const auto rounds = [&](int tiles) {
    return (((a.RB - 1) / tiles + 1) * blocks + kCus - 1) / kCus;
  };
  if (8 * rounds(16) < 5 * rounds(8)) return run_linear_g<TX, NT, 4 * NT, 2, 8, 1, GB>(a, s);
  return run_linear_g<TX, NT, 4 * NT, 2, 4, 2, GB>(a, s);
}

template <int GB>
hipError_t run_linear(const LinArgs& a, bool x_bf, hipStream_t s) {
  const int64_t tiles = (int64_t)a.RB * ((a.T + 15) / 16);
  const int64_t rows = (a.RB + 7) / 8, enough = kCus * 3 / 4;  // as above
  if constexpr (GB < 4) {
    if (x_bf && a.T > 32 && rows * ((a.T + 63) / 64) >= enough)
      return run_linear_wide<uint16_t, 4, GB>(a, s);
    if (!x_bf && a.T > 16 && rows * ((a.T + 31) / 32) >= enough)
      return run_linear_wide<float, 2, GB>(a, s);
  }
  // groups of 32 need more registers: 32 tokens and one row tile a wave (14336 x
  // 4096 at 64 tokens 43.9 us with 16 tokens, 27.3 so; fp32 91.1 and 61.0)
  if (a.T > 16 && rows * ((a.T + 31) / 32) >= enough) {
    if (x_bf) return run_linear_g<uint16_t, 2, 8, 1, 8, 2, GB>(a, s);
    if constexpr (GB == 4) return run_linear_g<float, 2, 8, 1, 4, 2, GB>(a, s);
  }
  // 64 rows by 32 tokens between the two, where one round of them covers more than
  // four tiles a CU (at 64 tokens, 4096 columns, 6144 rows: 11.5 us, with 16 tokens 12.3,
  // 8192 rows 11.8 and 12.5, groups of 64: 13.1 and 15.3, 13.4 and 15.5; 4096 rows, four
  // tiles a CU: 11.2 and 8.7)
  if constexpr (GB < 4)
    if (x_bf && a.T > 16 && tiles > 4 * kCus &&
        (int64_t)((a.RB + 3) / 4) * ((a.T + 31) / 32) <= kCus)
      return run_linear_g<uint16_t, 2, 8, 1, 4, 4, GB>(a, s);
  if (a.T <= 4) return x_bf ? run_linear_16<1, GB>(a, tiles, s) : run_linear_32<1, GB>(a, tiles, s);
  if (a.T <= 8) return x_bf ? run_linear_16<2, GB>(a, tiles, s) : run_linear_32<2, GB>(a, tiles, s);
  return x_bf ? run_linear_16<4, GB>(a, tiles, s) : run_linear_32<4, GB>(a, tiles, s);
}

}  // namespace

hipError_t launch_linear(const void* x, d2moe_dtype xd, int T, const d2moe_linear* w,
                         const float* bias, void* y, d2moe_dtype yd, hipStream_t s) {
  if (T == 0) return hipSuccess;
  const LinArgs a{x, w->codes, w->scales, w->zeros, bias, y, T, w->rows, w->cols,
                  lin_row_blocks(w), lin_col_blocks(w), yd == D2MOE_BF16};
  const bool x_bf = xd == D2MOE_BF16;
  return w->group == 128  ? run_linear<1>(a, x_bf, s)
         : w->group == 64 ? run_linear<2>(a, x_bf, s)
                          : run_linear<4>(a, x_bf, s);
}

}  // namespace d2moe
