// Attention of one new token per sequence over a paged key-value cache,
//   out[b][h] = sum_j softmax_j(scale q[b][h] . K_j) V_j,
// as one pass over the keys with the running maximum m, the sum l of
// exp(score - m) and the running value sum O, rescaled when m grows.
//
// The query heads of one key head (G of them, 16 at a time) are the columns of
// 16 x 16 matrix products, so a key or value row is read once for all of them:
//   S (keys x heads) = K Q^T,   O^T (values x heads) = V^T P^T.
// Both leave one head in lane column l % 16, and the four lanes of a column
// hold keys 4 q .. 4 q + 3 of a 16-key tile (q = l / 16).  The order of the
// keys in the second product is free, so its operand P^T takes exactly the
// keys that a lane computed, and V^T is read to match: no exchange between the
// products, only the maximum crosses lanes.
//
// The tiles of all sequences and key heads stand in one row that is cut into
// equal shares, one a workgroup, so that sequences of any lengths fill the chip
// evenly.  A share that holds a key head's tiles only in part leaves its m, l and
// O in the workspace, and a second kernel joins the parts.
//
// Bound by reading the cache: 4 len head_dim bytes (bf16) per key head against
// 16-column products that keep the matrix units busy for a twelfth of the time (64
// sequences of 8192 keys).
#include "decoder.h"

namespace d2moe {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int kHeadTile = 16;    // query heads of a workgroup
constexpr int kChunk = 512;      // keys whose row offsets are worked out at a time
// Units from which none is split: they are many a CU then, and one whole a workgroup
// is faster, with lengths near max_len (256 sequences of up to 4500 keys, 128 a head,
// 16 key heads: 831 us whole, 847 split, 32: 1600 and 1634, but 8: 441 and 429) and the
// more so below it (up to 1000 where 5000 are expected, 8 key heads: 107 and 139, up to
// 100: 20.6 and 49.5).  The price: one long sequence among short ones goes at the rate
// of one CU a key head (one of 32000, 255 of 300, 8 key heads: 435 and 106 us).
constexpr int kMaxSplitUnits = 2048;
constexpr int kSplitSeqs = 256;  // most sequences of a call whose keys are split
constexpr int kWholeBytes = 256 << 10;  // of keys: up to here a workgroup takes a unit whole
// Least tiles of a share, one a wave: with fewer more parts are joined, with more
// fewer CUs read (3000 keys of one head of 128: 11.1 us with 1, 9.6 with 4, 10.5 with 8;
// 4096 keys of 8 heads: 12.0 with 1 to 4, 12.2 with 8, 14.0 with 16).
constexpr int kMinShare = 4;
constexpr int kCus = 256;

struct AttnArgs {
  const void *q, *k, *v;
  int64_t q_stride, page_stride, token_stride, head_stride;
  const int32_t *table, *lengths;
  FastDiv page;
  int B, n_pages, max_pages, Hq, H, G, tiles, D, window, groups;
  float scale_log2;  // scale / ln 2
  void* out;
  float *part_o, *part_ml;  // [groups][2][min(G, 16)] rows of D and of 2
};

// Keys of sequence b that are attended: [first, first + count).
__device__ inline void key_range(const AttnArgs& a, int b, int& first, int& count) {
  int n = a.lengths[b];
  const int64_t room = (int64_t)a.max_pages * a.page.d;
  n = n < 0 ? 0 : n > room ? (int)room : n;
  first = a.window > 0 && n > a.window ? n - a.window : 0;
  count = n - first;
}

// Where the tiles of each sequence stand in the row of all: sequence b's units
// (key heads times head tiles, `per` of them) one after the other, t_b tiles each,
// from per * (t_0 + .. + t_{b-1}) on.  Held by every wave in its registers, lane
// l the sequences 4 l .. 4 l + 3.  (The host sees to it that the row has fewer
// than 2^31 tiles.)
struct Row {
  int upto[4];  // tiles of the sequences up to and with this one, one unit each
  int total;
};
__device__ inline Row row_of_tiles(const AttnArgs& a, int tk) {
  const int lane = threadIdx.x & 63;
  Row r;
  int sum = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    int first, count = 0;
    if (4 * lane + i < a.B) key_range(a, 4 * lane + i, first, count);
    sum += (count + tk - 1) / tk;
    r.upto[i] = sum;
  }
  int inc = sum;  // over the lanes: within rows of 16, then across the rows
  inc += __builtin_amdgcn_update_dpp(0, inc, 0x111, 0xf, 0xf, true);
  inc += __builtin_amdgcn_update_dpp(0, inc, 0x112, 0xf, 0xf, true);
  inc += __builtin_amdgcn_update_dpp(0, inc, 0x114, 0xf, 0xf, true);
  inc += __builtin_amdgcn_update_dpp(0, inc, 0x118, 0xf, 0xf, true);
  const int r0 = __builtin_amdgcn_readlane(inc, 15), r1 = __builtin_amdgcn_readlane(inc, 31),
            r2 = __builtin_amdgcn_readlane(inc, 47);
  inc += lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r0 + r1 : r0 + r1 + r2;
#pragma unroll
  for (int i = 0; i < 4; ++i) r.upto[i] += inc - sum;
  r.total = __builtin_amdgcn_readlane(inc, 63);
  return r;
}
__device__ inline int row_upto(const Row& r, int b) {  // uniform; 0 for b = -1
  if (b < 0) return 0;
  const int i = b & 3;
  return __builtin_amdgcn_readlane(
      i == 0 ? r.upto[0] : i == 1 ? r.upto[1] : i == 2 ? r.upto[2] : r.upto[3], b >> 2);
}
// Tiles of a share: the row in equal parts, but kMinShare at least.
__device__ inline int row_share(const Row& r, int per, int groups) {
  const int share = (int)(((int64_t)r.total * per + groups - 1) / groups);
  return share > kMinShare ? share : kMinShare;
}

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ inline f4 mma(u4 a, u4 b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                 __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));  // the result gets registers of its own
  return d;
}
__device__ inline f4 mma(float a, float b, f4 c) {
  f4 d = __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
  asm("" : "+v"(d) : "v"(a), "v"(b));
  return d;
}

// The tile products of one cache type: TK keys a step, a lane's share of the key
// rows as loaded (K), of the value rows (V) and of Q.  Head dimensions past D, where
// it is below DP (PAD), are zero in K and Q; value loads past D read the row's
// start and their results are not used.
//
// An operand of the key product has neighbouring lanes in neighbouring rows, and
// loads of that pattern take the L1 four times as long as loads of whole rows
// (a workgroup alone read 14 bytes a cycle).  Key rows are therefore loaded as
// they lie, CPR lanes of 16 bytes a row, and turned in LDS by the wave that uses
// them: chunk c of row r lies at r CPR + (c ^ swizzle(r)), so that 16 lanes meet 16
// different bank groups both writing (one row) and reading (16 rows, one c).
//
// Of a value row a lane loads VE consecutive values, dimensions 16 VE h + VE (l % 16)
// + 0 .. VE - 1, so that 16 lanes read a run of 16 VE values; element i of that run
// is the row l % 16 of value product (h, i).
template <int CPR>
__device__ inline int swizzle(int row) {
  return CPR >= 16 ? row & 15 : (row >> 1) & 7;
}

template <typename E, int DP, int TK_>
struct KeyRows {
  static constexpr int TK = TK_, PER = 16 / sizeof(E), CPR = DP / PER;
  static constexpr int NK = TK * CPR / 64, KS = CPR / 4;  // loads of a lane; operands of 16 rows
  struct K { u4 f[NK]; };
  struct Lds { u4 x[TK * CPR]; };
  static_assert(CPR >= 8 && TK * CPR % 64 == 0, "a load covers whole rows");

  template <bool PAD>
  __device__ static void load(K& o, const E* k, const int64_t* off, int lane, int D) {
#pragma unroll
    for (int j = 0; j < NK; ++j) {
      const int x = 64 * j + lane, row = x / CPR;
      int c = (x % CPR ^ swizzle<CPR>(row)) * PER;
      if (PAD && c >= D) c = 0;
      const int64_t at = off[row];
      o.f[j] = *(const u4*)(k + (at < 0 ? 0 : at) + c);
    }
  }
  __device__ static void store(Lds& l, const K& k, int lane) {
#pragma unroll
    for (int j = 0; j < NK; ++j) l.x[64 * j + lane] = k.f[j];
  }
  // operand s of tile t: row 16 t + l % 16, chunk 4 s + l / 16
  template <bool PAD>
  __device__ static u4 operand(const Lds& l, int t, int s, int lane, int D) {
    const int row = 16 * t + (lane & 15), c = 4 * s + (lane >> 4);
    const u4 v = l.x[row * CPR + (c ^ swizzle<CPR>(row))];
    return PAD && c * PER >= D ? u4{0, 0, 0, 0} : v;
  }
};

template <typename T, int DP, bool PAD>
struct Tile;

template <int DP, bool PAD>
struct Tile<uint16_t, DP, PAD> : KeyRows<uint16_t, DP, 32> {
  using Rows = KeyRows<uint16_t, DP, 32>;
  using typename Rows::Lds;
  static constexpr int VE = DP >= 128 ? 8 : 4, H = DP / (16 * VE), KS = Rows::KS;
  static constexpr int NV = 8;  // value rows (keys) of a lane
  struct Q { u4 f[KS]; };
  struct V { uint32_t f[NV][H][VE / 2]; };

  __device__ static int key_of(int j, int q) { return j < 4 ? 4 * q + j : 12 + 4 * q + j; }

  __device__ static void load_q(Q& o, const uint16_t* row, int q, int D, bool live) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 32 * s + 8 * q;
      o.f[s] = u4{0, 0, 0, 0};
      if (live && (!PAD || c < D)) o.f[s] = *(const u4*)(row + c);
    }
  }
  __device__ static void load_v(V& o, const uint16_t* v, const int64_t (&at)[NV], int lane, int D) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const uint16_t* row = v + (at[j] < 0 ? 0 : at[j]);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        int c = 16 * VE * h + VE * (lane & 15);
        if (PAD && c >= D) c = 0;
        if constexpr (VE == 8) {
          const u4 x = *(const u4*)(row + c);
#pragma unroll
          for (int d = 0; d < 4; ++d) o.f[j][h][d] = x[d];
        } else {
          const uint2 x = *(const uint2*)(row + c);
          o.f[j][h][0] = x.x;
          o.f[j][h][1] = x.y;
        }
      }
    }
  }
  __device__ static void clear_v(V& o, const int64_t (&at)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int d = 0; d < VE / 2; ++d) o.f[j][h][d] = at[j] < 0 ? 0u : o.f[j][h][d];
  }
  __device__ static void scores(float (&s)[NV], const Lds& k, const Q& q, int lane, int D) {
    u4 x[2][KS];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int c = 0; c < KS; ++c) x[t][c] = Rows::template operand<PAD>(k, t, c, lane, D);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int c = 0; c < KS; ++c) acc = mma(x[t][c], q.f[c], acc);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * t + i] = acc[i];
    }
  }
  // The probabilities enter as three bf16 pieces whose sum is exact (two would leave
  // an error of 2^-17 a key, some 14 times that of the binary32 sums).  Each of the first
  // two is the number below what is left, cut to its upper 16 bits, so that every
  // piece of a probability above zero is above zero and an infinite value stays one,
  // while a probability of zero adds nothing, whatever the value.  exp2 gives 0 or
  // 2^-126 and more; below 2^-103 the last pieces are denormals, which the products
  // take as they are, and no less than the least of those, 2^-133.  16 sequences of up
  // to 4096 keys, 8 heads of 128: 39.8 us with two pieces, 40.3 with three; 64 of up to
  // 2000, 4 heads of 256: 68.7 and 73.0; 16 of up to 2000, 8 of 64: 14.7 and 15.8; 64 of
  // 8192, 8 heads of 128: 377.5 both.
  __device__ static uint32_t upper(uint32_t second, uint32_t first) {
    return __builtin_amdgcn_perm(second, first, 0x07060302u);
  }
  __device__ static void values(f4 (&o)[H][VE], const float (&p)[NV], const V& v) {
    u4 piece[3];
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint32_t cut[3][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float all = p[2 * d + e];
        const int least = __builtin_elementwise_min(__float_as_uint(all), 0x10000u);
        cut[0][e] = __builtin_elementwise_sub_sat(__float_as_uint(all), 1u);
        const float rest = all - __uint_as_float(cut[0][e] & 0xffff0000u);
        const int next = __builtin_elementwise_sub_sat(__float_as_uint(rest), 1u);
        cut[1][e] = __builtin_elementwise_max(next, least);
        const int last = __float_as_int(rest - __uint_as_float(cut[1][e] & 0xffff0000u));
        cut[2][e] = __builtin_elementwise_max(last, least);
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) piece[k][d] = upper(cut[k][1], cut[k][0]);
    }
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < VE; ++i) {
        u4 a;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          a[d] = __builtin_amdgcn_perm(v.f[2 * d + 1][h][i / 2], v.f[2 * d][h][i / 2],
                                       (i & 1) ? 0x07060302u : 0x05040100u);
#pragma unroll
        for (int k = 0; k < 3; ++k) o[h][i] = mma(a, piece[k], o[h][i]);
      }
  }
};

template <int DP, bool PAD>
struct Tile<float, DP, PAD> : KeyRows<float, DP, 16> {
  using Rows = KeyRows<float, DP, 16>;
  using typename Rows::Lds;
  static constexpr int VE = 4, H = DP / 64, KS = Rows::KS;
  static constexpr int NV = 4;
  struct Q { f4 f[KS]; };
  struct V { f4 f[NV][H]; };

  __device__ static int key_of(int j, int q) { return 4 * q + j; }

  __device__ static void load_q(Q& o, const float* row, int q, int D, bool live) {
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      const int c = 16 * s + 4 * q;
      o.f[s] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      if (live && (!PAD || c < D)) o.f[s] = *(const f4*)(row + c);
    }
  }
  __device__ static void load_v(V& o, const float* v, const int64_t (&at)[NV], int lane, int D) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const float* row = v + (at[j] < 0 ? 0 : at[j]);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        int c = 64 * h + 4 * (lane & 15);
        if (PAD && c >= D) c = 0;
        o.f[j][h] = *(const f4*)(row + c);
      }
    }
  }
  __device__ static void clear_v(V& o, const int64_t (&at)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int e = 0; e < 4; ++e) o.f[j][h][e] = at[j] < 0 ? 0.0f : o.f[j][h][e];
  }
  __device__ static void scores(float (&s)[NV], const Lds& k, const Q& q, int lane, int D) {
    f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      const f4 x = __builtin_bit_cast(f4, Rows::template operand<PAD>(k, 0, c, lane, D));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f4 sum = mma(x[e], q.f[c][e], acc);
        // nor shares part of them with the sum so far
        if (c + e > 0) asm("" : "+v"(sum) : "v"(acc));
        acc = sum;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = acc[i];
  }
  __device__ static void values(f4 (&o)[H][VE], const float (&p)[NV], const V& v) {
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < VE; ++i)
#pragma unroll
        for (int j = 0; j < NV; ++j) o[h][i] = mma(v.f[j][h][i], p[j], o[h][i]);
  }
};

// A barrier for LDS alone: a full one would also wait for the loads under way.
__device__ inline void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// LDS between the lanes of a wave.
__device__ inline void wave_handoff() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Four values of a result row.
template <typename T>
__device__ inline void store4(T* p, f4 v) {
  if constexpr (sizeof(T) == 2)
    *(uint2*)p = make_uint2(f2bf(v[0]) | (uint32_t)f2bf(v[1]) << 16,
                            f2bf(v[2]) | (uint32_t)f2bf(v[3]) << 16);
  else
    *(f4*)p = v;
}

// WAVES waves take tiles of TK keys in turn; HT: query heads that the workgroup
// may have (4 or 16; columns past them are computed on zeros).  SPLIT: a
// workgroup takes its share of the row of tiles, otherwise one unit whole.
//
// The row offsets of the keys are worked out by all threads into LDS, so that no
// lookup in the block table stands between the loads of the loop.  The next
// tile's keys are loaded while this one's are used.  Every load of the loop is
// made, on whatever row where there is no key: a wait can then count on the loads
// behind the one it is for.
template <typename T, int DP, bool PAD, int HT, int WAVES, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, DP <= 128 ? 2 : 1) void attn_decode_kernel(AttnArgs a) {
  using M = Tile<T, DP, PAD>;
  struct Join {
    float m[WAVES][HT], l[WAVES][HT];
    __align__(16) float o[WAVES][HT][DP + 4];
  };
  struct Loop {
    int64_t off[3][kChunk];
    typename M::Lds k[WAVES];
  };
  union Lds {
    Loop loop;
    Join join;
  };
  __shared__ Lds lds;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, q = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int per = a.H * a.tiles;  // units of a sequence

  // tiles at .. end - 1 of the row, or the one unit
  Row row;
  int at = blockIdx.x, end = blockIdx.x + 1;
  if constexpr (SPLIT) {
    row = row_of_tiles(a, M::TK);
    const int share = row_share(row, per, a.groups);
    const int64_t to = ((int64_t)blockIdx.x + 1) * share, all = (int64_t)row.total * per;
    if (to - share >= all) return;
    at = (int)(to - share);
    end = (int)(to < all ? to : all);
  }
  while (at < end) {
    // the next segment: tiles j0 .. j1 - 1 of unit `unit` of sequence b
    int b, unit, j0 = 0, j1, seq_tiles, first, count;
    if constexpr (SPLIT) {
      b = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) b += __popcll(__ballot(row.upto[i] * per <= at));
      const int before = row_upto(row, b - 1);
      seq_tiles = row_upto(row, b) - before;
      const uint32_t in = at - before * per;
      unit = in / (uint32_t)seq_tiles;
      j0 = in - unit * seq_tiles;
      j1 = seq_tiles - j0 < end - at ? seq_tiles : j0 + (end - at);
      key_range(a, b, first, count);
    } else {
      b = at / per;
      unit = at - b * per;
      key_range(a, b, first, count);
      j1 = seq_tiles = (count + M::TK - 1) / M::TK;
    }
    const int hk = unit % a.H, tile = unit / a.H;
    const int g0 = tile * kHeadTile;                               // of the key head's G heads
    const int heads = a.G - g0 < kHeadTile ? a.G - g0 : kHeadTile;  // of this unit
    const int h0 = hk * a.G + g0;
    const T* kc = (const T*)a.k + hk * a.head_stride;
    const T* vc = (const T*)a.v + hk * a.head_stride;
    typename M::Q qf;
    M::load_q(qf, (const T*)a.q + b * a.q_stride + (int64_t)(h0 + (col < heads ? col : 0)) * a.D,
              q, a.D, col < heads);
    float m = -INFINITY, l = 0.0f;
    f4 o[M::H][M::VE];
#pragma unroll
    for (int h = 0; h < M::H; ++h)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) o[h][i] = f4{0.0f, 0.0f, 0.0f, 0.0f};

    // Row offsets (-1: masked) by all threads, kChunk keys at a time: chunk c's
    // lie at c % 3, are written a chunk before they are first used, and their
    // block-table entries are read a chunk before that.
    constexpr int kTiles = kChunk / M::TK, kEach = kChunk / (64 * WAVES);
    static_assert(kTiles % WAVES == 0 && kChunk % (64 * WAVES) == 0, "whole tiles and threads");
    const int n_tiles = j1 - j0, s0 = j0 * M::TK;
    const int chunks = (n_tiles + kTiles - 1) / kTiles;
    auto fetch = [&](int c, int (&page)[kEach]) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const uint32_t at = a.page.div(first + s0 + c * kChunk + e * 64 * WAVES + tid);
        page[e] = a.table[(int64_t)b * a.max_pages +
                          (at < (uint32_t)a.max_pages ? at : (uint32_t)a.max_pages - 1)];
      }
    };
    auto put = [&](int c, const int (&page)[kEach]) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) {
        const int i = e * 64 * WAVES + tid, at = s0 + c * kChunk + i;
        const uint32_t key = (uint32_t)(first + at);
        const bool in = at < count && (uint32_t)page[e] < (uint32_t)a.n_pages;
        lds.loop.off[c % 3][i] =
            in ? page[e] * a.page_stride +
                     (int64_t)(key - a.page.div(key) * a.page.d) * a.token_stride
               : -1;
      }
    };
    int page[kEach];
    if (n_tiles > 0) {
      int page0[kEach];
      fetch(0, page0);
      if (chunks > 1) fetch(1, page);
      lds_barrier();  // what was there has been used
      put(0, page0);
      if (chunks > 1) put(1, page);
      lds_barrier();
    }
    typename M::K kf;
    auto offsets = [&](int t) { return &lds.loop.off[t / kTiles % 3][t % kTiles * M::TK]; };
    int t = wave;
    if (t < n_tiles) M::template load<PAD>(kf, kc, offsets(t), lane, a.D);
    for (int c = 0; c < chunks; ++c) {
      if (c > 0) {
        if (c + 1 < chunks) put(c + 1, page);
        lds_barrier();  // and chunk c - 1 has been used
      }
      if (c + 2 < chunks) fetch(c + 2, page);
      const int stop = n_tiles < (c + 1) * kTiles ? n_tiles : (c + 1) * kTiles;
      for (; t < stop; t += WAVES) {
        const int64_t* off = offsets(t);
        int64_t from[M::NV];
#pragma unroll
        for (int j = 0; j < M::NV; ++j) from[j] = off[M::key_of(j, q)];
        typename M::V vf;
        M::load_v(vf, vc, from, lane, a.D);
        M::store(lds.loop.k[wave], kf, lane);
        M::template load<PAD>(kf, kc, offsets(t + WAVES < n_tiles ? t + WAVES : t), lane, a.D);
        wave_handoff();
        float s[M::NV];
        M::scores(s, lds.loop.k[wave], qf, lane, a.D);
        wave_handoff();
        bool hole = false;
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < M::NV; ++j) {
          s[j] = from[j] < 0 ? -INFINITY : s[j] * a.scale_log2;
          hole |= from[j] < 0;
          mx = fmaxf(mx, s[j]);
        }
        mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float m_new = fmaxf(m, mx);
        const float ref = m_new == -INFINITY ? 0.0f : m_new;  // nothing but masked keys so far
        const float alpha = fast_exp2(m - ref);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int j = 0; j < M::NV; ++j) {
          s[j] = fast_exp2(s[j] - ref);
          l += s[j];
        }
        if (__any(alpha != 1.0f)) {
#pragma unroll
          for (int h = 0; h < M::H; ++h)
#pragma unroll
            for (int i = 0; i < M::VE; ++i) o[h][i] *= alpha;
        }
        if (__any(hole)) M::clear_v(vf, from);  // 0 times what a masked row holds is not 0
        M::values(o, s, vf);
      }
    }

    // join the waves: every head's m, l and O
    lds_barrier();  // the offsets have been used
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (col < HT) {
      if (q == 0) {
        lds.join.m[wave][col] = m;
        lds.join.l[wave][col] = l;
      }
#pragma unroll
      for (int h = 0; h < M::H; ++h)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
          for (int i = 0; i < M::VE; i += 4)
            *(f4*)&lds.join.o[wave][col][16 * M::VE * h + M::VE * (4 * q + r) + i] =
                f4{o[h][i][r], o[h][i + 1][r], o[h][i + 2][r], o[h][i + 3][r]};
    }
    lds_barrier();
    const int row4 = a.D / 4;
    for (int i = tid; i < heads * row4; i += 64 * WAVES) {
      const int g = i / row4, d = (i - g * row4) * 4;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) mm = fmaxf(mm, lds.join.m[w][g]);
      const float ref = mm == -INFINITY ? 0.0f : mm;
      float ll = 0.0f;
      f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int w = 0; w < WAVES; ++w) {
        const float f = fast_exp2(lds.join.m[w][g] - ref);
        ll = fmaf(f, lds.join.l[w][g], ll);
        acc += f * *(const f4*)&lds.join.o[w][g][d];
      }
      if (SPLIT && j1 - j0 < seq_tiles) {
        // a share has one part at most that begins a unit and one that does not
        const int rows = a.G < kHeadTile ? a.G : kHeadTile;
        const int64_t to = ((int64_t)blockIdx.x * 2 + (j0 > 0 ? 0 : 1)) * rows + g;
        *(f4*)(a.part_o + to * a.D + d) = acc;
        if (d == 0) *(float2*)(a.part_ml + to * 2) = make_float2(mm, ll);
      } else {
        store4((T*)a.out + ((int64_t)b * a.Hq + h0 + g) * a.D + d,
               acc * (ll == 0.0f ? 0.0f : 1.0f / ll));
      }
    }
    if constexpr (SPLIT) at += j1 - j0;
    else at = end;
  }
}

// Joins the parts of one query head: the waves (a lane has four values) take
// parts in turn.  A unit that one share holds whole is done already, one without
// keys gives zeros.
template <typename T, int TK, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attn_join_kernel(AttnArgs a) {
  __shared__ float pm[WAVES], pl[WAVES];
  __shared__ __align__(16) f4 po[WAVES][64];
  const int b = blockIdx.y, head = blockIdx.x;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int per = a.H * a.tiles, rows = a.G < kHeadTile ? a.G : kHeadTile;
  const int hk = head / a.G, tile = (head - hk * a.G) / kHeadTile;
  const int g = head - hk * a.G - tile * kHeadTile;
  const Row row = row_of_tiles(a, TK);
  const int share = row_share(row, per, a.groups);
  const int before = row_upto(row, b - 1), tiles = row_upto(row, b) - before;
  const int from = before * per + (tile * a.H + hk) * tiles;
  const int w0 = from / share, n = tiles == 0 ? 0 : (from + tiles - 1) / share - w0 + 1;
  if (n == 1) return;
  const int d = 4 * lane < a.D ? 4 * lane : 0;
  // part i lies in share w0 + i; the first begins the unit
  auto part = [&](int i) { return ((int64_t)(w0 + i) * 2 + (i == 0 ? 1 : 0)) * rows + g; };
  float mm = -INFINITY, ll = 0.0f;
  f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int kAhead = 4;  // parts loaded together
  for (int i = wave; i < n; i += kAhead * WAVES) {
    float2 ml[kAhead];
    f4 v[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t p = part(i + k * WAVES < n ? i + k * WAVES : i);
      ml[k] = *(const float2*)(a.part_ml + p * 2);
      v[k] = *(const f4*)(a.part_o + p * a.D + d);
    }
    float top = mm;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) top = fmaxf(top, ml[k].x);
    const float ref = top == -INFINITY ? 0.0f : top, alpha = fast_exp2(mm - ref);
    mm = top;
    ll *= alpha;
    acc *= alpha;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (i + k * WAVES >= n) break;
      const float f = fast_exp2(ml[k].x - ref);
      ll = fmaf(f, ml[k].y, ll);
      acc += f * v[k];
    }
  }
  po[wave][lane] = acc;
  if (lane == 0) pm[wave] = mm, pl[wave] = ll;
  __syncthreads();
  if (wave != 0 || 4 * lane >= a.D) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w) mm = fmaxf(mm, pm[w]);
  const float ref = mm == -INFINITY ? 0.0f : mm;
  ll = 0.0f;
  acc = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    const float f = fast_exp2(pm[w] - ref);
    ll = fmaf(f, pl[w], ll);
    acc += f * po[w][lane];
  }
  store4((T*)a.out + ((int64_t)b * a.Hq + head) * a.D + d,
         acc * (ll == 0.0f ? 0.0f : 1.0f / ll));
}

int head_tiles(int q_heads, int n_heads) {
  return (q_heads / n_heads + kHeadTile - 1) / kHeadTile;
}

int head_units(int B, int q_heads, int n_heads) {
  return B * n_heads * head_tiles(q_heads, n_heads);  // at most B * q_heads, 2^22, checked first
}

// Workgroups of a call whose keys are split: one per CU, whose four waves keep
// enough loads under way (1 sequence of 32768 keys, 8 heads of 128: 32.7 us, with
// two 33.7; 64 ragged ones of up to 8192: 252 us = 5.5 TB/s, with two 261); two
// where the units are many and short, so that one's start and end lie under the
// other's loads (32 sequences of up to 2000 keys, 40 heads: 133 and 125 us), or the
// rows short (64 of up to 2000, 8 heads of 64: 46.5 and 36.8).  Eight waves a workgroup
// were no faster (with two pieces of the probabilities: 249 us against 251, 4096 keys of
// one sequence 13.2 against 12.7).
int split_groups(int units, int dim) {
  return kCus * (dim <= 64 || (dim <= 128 && units > 512) ? 2 : 1);
}

// Whether the keys are split.  Not where a second kernel, the look over all lengths
// and a cold start of every share cost more than the split saves: up to 256 KB of keys
// a unit (16 sequences of up to 1000 keys, 8 heads of 128, bf16: whole 14.0 us, split
// 19.1, up to 2000: 23.1 and 21.2; 64 a head, up to 2000: 15.6 and 15.8, up to 3000: 21.8
// and 20.4; fp32, 16 of up to 1000, 64 a head: 16.9 and 17.3, up to 1500: 23.4 and 19.5),
// twice that in bf16 where the units fill the chip by themselves (64 of up to 1500,
// 8 heads of 128: 47.2 and 57.8, but 32 of up to 4096: 71.4 and 63.2; fp32, whose units
// take longer: 64 of up to 2000, 12 heads of 64: 94.0 and 80.5).  Nor where a row of
// tiles could pass 2^31.
bool attn_splits(int B, int q_heads, int n_heads, int dim, int size, int keys, int64_t room) {
  if (B > kSplitSeqs) return false;
  const int64_t units = head_units(B, q_heads, n_heads);
  const int64_t unit_bytes = (int64_t)keys * size * (dim <= 64 ? 64 : dim <= 128 ? 128 : 256);
  return unit_bytes > (size == 2 && units > kCus ? 2 : 1) * kWholeBytes &&
         units < kMaxSplitUnits &&
         units * ((room < 0x7fffffff ? room : 0x7fffffff) / 16 + 1) < 0x7fffffff;
}

// Waves of a workgroup that takes a unit whole: eight where the chip has room for
// them, two where units are many and short, so that more of them are under way (up to
// 64 keys, 8 heads of 128, bf16, 128 sequences: 10.7 us with four, 7.9 with two, 2000
// sequences of up to 200 225 and 189; but 64 sequences, two units a CU, of up to 500
// 17.8 and 19.3, and 300 with 4 heads of up to 3000 208 both; fp32, 128 sequences, 12
// heads of 64: 64 keys 11.5 and 10.7, 220 keys 22.8 and 25.0).
template <typename T, int DP, bool PAD, int HT>
void run_attn_h(const AttnArgs& a, bool split, int keys, hipStream_t s) {
  const int units = a.B * a.H * a.tiles;
  const bool short_units =
      (int64_t)keys * DP * sizeof(T) <= (sizeof(T) == 2 ? kWholeBytes / 2 : kWholeBytes / 8);
  if (split)
    attn_decode_kernel<T, DP, PAD, HT, 4, true><<<a.groups, 256, 0, s>>>(a);
  else if (DP <= 128 && units <= kCus)
    attn_decode_kernel<T, DP, PAD, HT, DP <= 128 ? 8 : 4, false><<<units, 512, 0, s>>>(a);
  else if (units > 2 * kCus && short_units)
    attn_decode_kernel<T, DP, PAD, HT, 2, false><<<units, 128, 0, s>>>(a);
  else
    attn_decode_kernel<T, DP, PAD, HT, 4, false><<<units, 256, 0, s>>>(a);
}

template <typename T, int DP, bool PAD>
hipError_t run_attn(const AttnArgs& a, bool split, int keys, hipStream_t s) {
  if (a.G <= 4)
    run_attn_h<T, DP, PAD, 4>(a, split, keys, s);
  else
    run_attn_h<T, DP, PAD, 16>(a, split, keys, s);
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess || !split) return err;
  constexpr int TK = Tile<T, DP, PAD>::TK;
  // 16 waves for many parts a unit (100000 keys of one key head: 21.7 us for both
  // kernels, with four waves 33.0; 32 parts: 12.0 and 13.0), four for few (16 sequences
  // of up to 4096 keys, 8 heads of 128: 40.0 us, with sixteen 41.4)
  if (a.groups >= 16 * a.B * a.H * a.tiles)
    attn_join_kernel<T, TK, 16><<<dim3(a.Hq, a.B), 1024, 0, s>>>(a);
  else
    attn_join_kernel<T, TK, 4><<<dim3(a.Hq, a.B), 256, 0, s>>>(a);
  return hipGetLastError();
}

// Dimensions between two widths load the row's start again for what is missing, from the
// L1 (64 sequences of up to 4000 keys, 8 heads of 64: 74 us, 80: 104, 96: 106, 112: 130,
// 128: 123; by their bytes, 80 would take 77 and 96 92 of the 123).
template <typename T>
hipError_t run_attn_t(const AttnArgs& a, bool split, int keys, hipStream_t s) {
  if (a.D == 64) return run_attn<T, 64, false>(a, split, keys, s);
  if (a.D < 64) return run_attn<T, 64, true>(a, split, keys, s);
  if (a.D == 128) return run_attn<T, 128, false>(a, split, keys, s);
  if (a.D < 128) return run_attn<T, 128, true>(a, split, keys, s);
  if (a.D == 256) return run_attn<T, 256, false>(a, split, keys, s);
  return run_attn<T, 256, true>(a, split, keys, s);
}

}  // namespace

size_t attn_decode_workspace(int B, int q_heads, int n_heads, int dim, int max_len) {
  // (fp32 caches, the first to be split)
  if (B == 0 || !attn_splits(B, q_heads, n_heads, dim, 4, max_len, 0)) return 0;
  const int rows = q_heads / n_heads < kHeadTile ? q_heads / n_heads : kHeadTile;
  return (size_t)split_groups(head_units(B, q_heads, n_heads), dim) * 2 * rows * (dim + 2) *
         sizeof(float);
}

hipError_t launch_attn_decode(const void* q, int64_t q_stride, int B, int q_heads,
                              const d2moe_kv_cache* c, const int32_t* table, int max_pages,
                              const int32_t* lengths, int max_len, int window, float scale,
                              void* out, void* ws, hipStream_t s) {
  if (B == 0) return hipSuccess;
  AttnArgs a{};
  a.q = q, a.k = c->k, a.v = c->v, a.q_stride = q_stride, a.page_stride = c->page_stride;
  a.token_stride = c->token_stride, a.head_stride = c->head_stride;
  a.table = table, a.lengths = lengths, a.page = fast_div(c->page_size);
  a.B = B, a.n_pages = c->n_pages, a.max_pages = max_pages, a.Hq = q_heads, a.H = c->n_heads;
  a.G = q_heads / c->n_heads, a.tiles = head_tiles(q_heads, c->n_heads), a.D = c->head_dim;
  a.window = window;
  const int keys = window > 0 && window < max_len ? window : max_len;
  const bool split = attn_splits(B, q_heads, c->n_heads, a.D, c->dtype == D2MOE_BF16 ? 2 : 4, keys,
                                 (int64_t)max_pages * c->page_size);
  a.groups = split_groups(head_units(B, q_heads, c->n_heads), a.D);
  a.scale_log2 = scale * kLog2e;
  a.out = out;
  const int rows = a.G < kHeadTile ? a.G : kHeadTile;
  a.part_o = (float*)ws;
  a.part_ml = (float*)ws + (size_t)a.groups * 2 * rows * a.D;
  return c->dtype == D2MOE_BF16 ? run_attn_t<uint16_t>(a, split, keys, s)
                                : run_attn_t<float>(a, split, keys, s);
}

}  // namespace d2moe
