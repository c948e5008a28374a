// w4.hip -- products of a few rows with 4-bit weights and group scales.
//
//   y[m, n] = b[n] + sum_g s[g, n] sum_{k in group g} x[m, k] (c[k, n] - z[g, n])
//
// for codes c in 0..15: the output layer of a drafting model, or any matrix
// whose bytes are what a product of few rows costs.
//
// Codes are packed by tiles of 16 columns x 128 rows, 1 KB each, all row
// blocks of a column tile after one another: 16-byte vector 16 q + r of a
// tile belongs to column r, its 32-bit word s to rows 32 s + 8 q .. + 7 of the
// block, nibble p of the word to row 2p (p < 4) or 2(p - 4) + 1.  Scales and
// zero points go with the tiles, [tile][row block][16][gpb]: gpb = 4, 2 or 1
// for groups of whole 32s, 64s or 128s of rows (a group's scale stands once
// for each of them), zeros past the last row.
#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>

#include "draft.hpp"

using namespace nmt;

constexpr int kW4Cols = 16, kW4Rows = 128;  // columns and rows of a packed tile
constexpr float kMostScale = 0x1p116f;      // the largest scale that products take

struct nmt_w4 {
  nmt_w4_dims dims{};
  int device = 0, cus = 0;
  int tiles = 0, kblocks = 0, gpb = 1;
  void* mem = nullptr;  // everything below
  uint4* codes = nullptr;
  void* scales = nullptr;  // fp32 or bf16
  uint8_t* zeros = nullptr;  // null: 8
  float* bias = nullptr;     // null: none
};

namespace {

__host__ __device__ inline int nibble_row(int p) { return p < 4 ? 2 * p : 2 * (p - 4) + 1; }

// ------------------------------------------------------------- packing

// One packed vector per thread, from row-major codes, two columns a byte.
__global__ __launch_bounds__(256) void k_w4_pack(const uint8_t* __restrict__ src, int K, int N, int kblocks,
                                                 int64_t n_all, uint4* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_all) return;
  const int lane = (int)(i & 63), r = lane & 15, q = lane >> 4;
  const int64_t tb = i >> 6, tile = tb / kblocks;
  const int kb = (int)(tb % kblocks);
  const int64_t n = tile * kW4Cols + r, stride = ((int64_t)N + 1) / 2;
  uint32_t w[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    w[s] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int k = kb * kW4Rows + s * 32 + q * 8 + nibble_row(p);
      const uint32_t c = (k < K && n < N) ? (src[(int64_t)k * stride + n / 2] >> (n & 1 ? 4 : 0)) & 15u : 0u;
      w[s] |= c << (4 * p);
    }
  }
  out[i] = uint4{w[0], w[1], w[2], w[3]};
}

// Where entry i of the scales belongs: its column, and its first row.
struct ScaleAt {
  int64_t n;
  int k;
};
__device__ __forceinline__ ScaleAt scale_at(int64_t i, int kblocks, int gpb) {
  const int64_t tb = i / (kW4Cols * gpb);
  return ScaleAt{tb / kblocks * kW4Cols + i / gpb % kW4Cols,
                 (int)(tb % kblocks) * kW4Rows + (int)(i % gpb) * (kW4Rows / gpb)};
}

// Scales (fp32 to ST, nearest even), zero points and bias into their places;
// zeros past the last column and row.
template <class ST>
__global__ __launch_bounds__(256) void k_w4_params(const float* __restrict__ scales, const uint8_t* __restrict__ zeros,
                                                   const float* __restrict__ bias, int K, int N, int group, int kblocks,
                                                   int gpb, int64_t n_all, ST* __restrict__ s_out,
                                                   uint8_t* __restrict__ z_out, float* __restrict__ b_out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_all) return;
  const ScaleAt at = scale_at(i, kblocks, gpb);
  const bool in = at.n < N && at.k < K;
  const int64_t from = in ? (int64_t)(at.k / group) * N + at.n : 0;
  s_out[i] = (ST)(in ? scales[from] : 0.f);
  if (zeros) z_out[i] = in ? zeros[from] : 0;
  if (bias && at.k == 0) b_out[at.n] = at.n < N ? bias[at.n] : 0.f;
}

// A model's output weight (k, n) from its packed matrix.
__device__ __forceinline__ float out_weight(const void* W, bool bf16, int64_t Npad, int k, int64_t n) {
  return bf16 ? (float)((const __bf16*)W)[((int64_t)(k / 8) * Npad + n) * 8 + k % 8]
              : ((const float*)W)[((int64_t)(k / 4) * Npad + n) * 4 + k % 4];
}

// Scales of the model's columns, one thread an entry: the group's largest
// magnitude / 7.
template <class ST>
__global__ __launch_bounds__(256) void k_w4_out_scales(const void* __restrict__ W, int bf16, int64_t Npad, int K, int N,
                                                       int group, int kblocks, int gpb, int krow, int nbias,
                                                       int64_t n_all, ST* __restrict__ s_out, float* __restrict__ b_out,
                                                       int* __restrict__ bad) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_all) return;
  const ScaleAt at = scale_at(i, kblocks, gpb);
  float mx = 0.f;
  bool finite = true;
  if (at.n < N) {
    const int k0 = at.k / group * group, k1 = at.k < K ? min(K, k0 + group) : 0;
    for (int k = k0; k < k1; ++k) {
      const float a = fabsf(out_weight(W, bf16, Npad, k, at.n));
      finite = finite && a < INFINITY;
      mx = fmaxf(mx, a);
    }
  }
  if (at.k == 0) {
    float b = 0.f;
    for (int j = 0; j < nbias && at.n < N; ++j) b += out_weight(W, bf16, Npad, krow + j, at.n);
    b_out[at.n] = b;
  }
  s_out[i] = (ST)(mx / 7.f);
  if (!finite || !(mx / 7.f <= kMostScale)) atomicOr(bad, finite ? 2 : 1);
}

// The codes under those scales, one packed vector per thread.
template <class ST>
__global__ __launch_bounds__(256) void k_w4_out_codes(const void* __restrict__ W, int bf16, int64_t Npad, int K, int N,
                                                      int kblocks, int gpb, int64_t n_all,
                                                      const ST* __restrict__ scales, uint4* __restrict__ out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_all) return;
  const int lane = (int)(i & 63), r = lane & 15, q = lane >> 4;
  const int64_t tb = i >> 6, tile = tb / kblocks;
  const int kb = (int)(tb % kblocks);
  const int64_t n = tile * kW4Cols + r;
  uint32_t w[4];
#pragma unroll
  for (int s = 0; s < 4; ++s) {
    w[s] = 0;
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      const int k = kb * kW4Rows + s * 32 + q * 8 + nibble_row(p);
      uint32_t c = 8;
      if (k < K && n < N) {
        const float sc = (float)scales[(tb * kW4Cols + r) * gpb + s * gpb / 4];
        const float v = sc != 0.f ? rintf(out_weight(W, bf16, Npad, k, n) / sc) : 0.f;
        c = (uint32_t)(8 + (int)fminf(fmaxf(v, -7.f), 7.f));
      }
      w[s] |= c << (4 * p);
    }
  }
  out[i] = uint4{w[0], w[1], w[2], w[3]};
}

// ------------------------------------------------------------- product
//
// On the fp16 matrix cores: codes minus their zero point are whole numbers of
// at most 15, exact in fp16, and the inputs enter as fp16 times a power of two,
// an fp32 input as two halves hi = fp16(x 2^e) and lo = fp16(x 2^e - hi), 22
// bits and a sign, a bf16 input as one.  e puts the largest of a row's 128
// inputs of a K block in [2^14, 2^15), so an input is off by at most 2^-23 of
// itself (a bf16 one by nothing) or 2^-39 of that largest one.  A group's
// products are summed in fp32 by the MFMA, then times the scale to the block's
// sum and times 2^(14 - e) to the row's, for the codes enter as c 2^-14.  With
// those a block's sum is below 128 * 15 * 2^15 * 2^-14 < 2^11.91 of its scales,
// so it cannot overflow before 2^-e is taken off while the scales are at most
// kMostScale, and 2^(14 - e) is a normal float for inputs of any size; whole
// codes would do for scales up to 2^102 alone.  (Scales below 2^-111 lose bits
// on the way, but fewer than the inputs' 2^-39.)
//
// A block takes up to RM rows, holds their inputs in LDS as MFMA fragments,
// converted once a block (K too long for LDS is taken in chunks), and walks over
// the column tiles, one for each group of WK waves at a time.  The codes stream
// from memory straight into registers, D K blocks ahead and from before the
// inputs are converted, each 16-byte vector the operand of four MFMA steps of
// 32 rows of W: 9 instructions turn a 32-bit word into eight fp16 values (the
// old way of making floats of small whole numbers, by putting them into the
// last bits of a known one: 0x2c00 | n is 2^-4 + n 2^-14; the upper nibble of a
// byte, in place, gives 2^-4 + n 2^-10).  Lane 16 q + r holds column r of a tile, so it needs one scale
// and one zero point a group.  WK > 1 splits K between waves where there are
// few columns; their sums meet in LDS in a fixed order.
//
// Measured, a call: 1 row of K = 500, N = 100,000 9.5 us (29 MB; its loads
// alone 5.5), 12 rows of N = 50,000 in groups of 32 8.0, 4 bf16 rows of 4096 x
// 4096 6.0, 32 inputs to 1,000 outputs 4.2 on the GPU: launch, first loads and
// the inputs' conversion.  80 rows of N = 100,000 30 us, bound by what the
// SIMDs issue: 114 VALU instructions beside the 16 MFMA steps of 32 rows x 16
// columns x 128 (16.7 us; the loads alone 9.5, staging 2.5, stores 4).
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

struct W4Args {
  const uint4* codes;
  const void* scales;
  const uint8_t* zeros;
  const float* bias;
  int K, N, kblocks, tiles, M;
  int y16;
  const void* x;
  int64_t ld_x;
  void* y;
  int64_t ld_y;
};
// How a launch is cut: rows a block (at most RM), row blocks, blocks that share
// a row block's columns (a multiple of 8), waves that share a column's K, K
// blocks a chunk (a multiple of D wk, or all).
struct W4Shape {
  int rows, row_blocks, strips, wk, chunk;
};
// Waves a block, and K blocks in flight.  Many rows, or a K that is long for 16
// rows, fill a CU's LDS by themselves, so their block is 16 waves (80 rows of K
// = 500, N = 100,000: 30 us, and 1.6 times that with 8); the others leave room for two
// blocks, and a wave for the whole K of an output layer (33 rows of 1001 x
// 7777: 10.1 us with two K blocks in flight, 9.1 with four).
constexpr int w4_waves(int RM, bool long_k) { return RM > 16 || (RM == 16 && long_k) ? 16 : 8; }
constexpr int w4_depth(int RM, int W, int GPB) { return W > 8 || (RM == 16 && GPB == 4) ? 2 : 4; }

// Eight codes of a word as fp16, minus the zero point, times 2^-14: zl = -(2^-4
// + z 2^-14) and zh = -(2^-8 + z 2^-14), twice each.  (The masks sit in registers, or the compiler
// splits each and-or for the sake of its literals.)
struct Masks {
  uint32_t lo = 0x000f000fu, hi = 0x00f000f0u, base = 0x2c002c00u;
  __device__ __forceinline__ Masks() { asm("" : "+s"(lo), "+s"(hi), "+v"(base)); }
};
__device__ __forceinline__ f16x8 codes_f16(uint32_t w, f16x2 zl, f16x2 zh, const Masks& k) {
  const f16x2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
  auto h2 = [](uint32_t u) { return __builtin_bit_cast(f16x2, u); };
  const uint32_t w8 = w >> 8;
  const f16x2 a = h2((w & k.lo) | k.base) + zl;
  const f16x2 b = __builtin_elementwise_fma(h2((w & k.hi) | k.base), sixteenth, zh);
  const f16x2 c = h2((w8 & k.lo) | k.base) + zl;
  const f16x2 d = __builtin_elementwise_fma(h2((w8 & k.hi) | k.base), sixteenth, zh);
  return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Eight consecutive inputs, those from n on as zeros; any alignment of the
// elements' own.
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
__device__ __forceinline__ void load8(const float* x, int n, float (&v)[8]) {
  if (n >= 8) {
    const f32x4u a = *(const f32x4u*)x, b = *(const f32x4u*)(x + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < 4 ? a[e] : b[e - 4];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? x[e] : 0.f;
  }
}
__device__ __forceinline__ void load8(const __bf16* x, int n, float (&v)[8]) {
  if (n >= 8) {
    const bf16x8u a = *(const bf16x8u*)x;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < n ? (float)x[e] : 0.f;
  }
}

// The largest magnitude of 16 consecutive lanes' eight values, as a float's
// bits (a NaN's lie above infinity's).
__device__ __forceinline__ uint32_t largest16(const float (&v)[8]) {
  float f = __builtin_elementwise_maximum(fabsf(v[0]), fabsf(v[1]));  // (NaN if either is)
#pragma unroll
  for (int e = 2; e < 8; ++e) f = __builtin_elementwise_maximum(f, fabsf(v[e]));
  uint32_t m = __builtin_bit_cast(uint32_t, f) & 0x7fffffffu;
  auto with = [&](auto ctrl) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, decltype(ctrl)::value, 0xf, 0xf, true));
  };
  with(std::integral_constant<int, 0xB1>{});   // lane ^ 1
  with(std::integral_constant<int, 0x4E>{});   // lane ^ 2
  with(std::integral_constant<int, 0x141>{});  // 7 - lane of 8
  with(std::integral_constant<int, 0x140>{});  // 15 - lane of 16
  return m;
}

template <int RM, int W, int GPB, bool X16, bool S16>
__global__ __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(4))) void k_w4_product(
    W4Args a, W4Shape sh) {
  constexpr int RT = (RM + 15) / 16;  // row tiles
  constexpr int HV = X16 ? 1 : 2;  // fp16 parts of an input
  constexpr int D = w4_depth(RM, W, GPB);
  using XT = std::conditional_t<X16, __bf16, float>;
  using ST = std::conditional_t<S16, __bf16, float>;
  // [K block][step][part][lane quarter][row ^ (4 step + quarter)] fragments
  // (rows permuted within their tile, so that the 16 lanes that write one
  // row's vectors do not meet in one bank; RM = 4 keeps them in order), then
  // [K block][16 RT] 2^(14 - e), then the K shares' sums
  extern __shared__ f32x4 lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, q = lane >> 4;
  // the row blocks of the same columns run on one XCD, whose L2 then holds their codes
  const int id = blockIdx.x, slot = id >> 3;
  const int strip = (slot / sh.row_blocks) * 8 + (id & 7), rb = slot % sh.row_blocks;
  const int wk = wave % sh.wk, per_block = W / sh.wk;  // tiles
  const int row0 = rb * sh.rows, rows = min(sh.rows, a.M - row0);

  // a K block's codes, scales and zero points, as they are in memory
  typedef ST scales_t __attribute__((ext_vector_type(GPB)));
  using zeros_t = std::conditional_t<GPB == 4, uint32_t, std::conditional_t<GPB == 2, uint16_t, uint8_t>>;
  struct Block {
    uint4 code;
    scales_t scale;
    zeros_t zero;
  };
  // Loads without a branch, or the compiler cannot tell how many are under way
  // and waits for all: past the end the last block is read once more, and
  // without zero points, in their place, bytes of the scales.
  const zeros_t* zeros = (const zeros_t*)(a.zeros ? (const void*)a.zeros : a.scales);
  auto load = [&](Block& b, int tile, int kb) {
    const int64_t tb = (int64_t)min(tile, a.tiles - 1) * a.kblocks + min(kb, a.kblocks - 1);
    b.code = (a.codes + tb * 64)[lane];
    b.scale = ((const scales_t*)a.scales + tb * kW4Cols)[r16];
    b.zero = (zeros + tb * kW4Cols)[r16];
  };
  // tiles go round the strips, then their waves: what is left in the last round
  // falls on one wave of many CUs, not on all of a few
  const int tile_step = sh.strips * per_block;
  int tile = strip + wave / sh.wk * sh.strips;
  Block ring[D];
#pragma unroll
  for (int d = 0; d < D; ++d) load(ring[d], tile, d * sh.wk + wk);

  // Eight inputs of a K block that 16 lanes hold to LDS; returns the block's 2^(14 - e)
  auto convert = [&](const float (&v)[8], f32x4* to) {
    constexpr uint32_t kInf = 0x7f800000u;
    uint32_t mx = largest16(v);  // (a NaN makes all of its row's outputs NaN, at any scale)
    const bool infinite = __ballot(mx == kInf) != 0;
    if (infinite) {  // the largest of the finite ones
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = fabsf(v[e]) < INFINITY ? v[e] : 0.f;
      mx = largest16(w);
    }
    // 2^e puts the largest in [2^14, 2^15); e not above 127, so that 2^e is finite (at 127 the halves still
    // hold every bit of fp32's smallest values, whose steps are 2^-149)
    const int e2 = mx - 1 < kInf - 1 ? min(15 - __builtin_amdgcn_frexp_expf(__builtin_bit_cast(float, mx)), 127) : 0;
    const float up = __builtin_amdgcn_ldexpf(1.f, e2);
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      hi[e] = (_Float16)(v[e] * up);
      if constexpr (HV == 2) lo[e] = (_Float16)fmaf(v[e], up, -(float)hi[e]);
    }
    if constexpr (HV == 2)
      if (infinite)  // an infinity is all in hi (inf - inf is no remainder)
#pragma unroll
        for (int e = 0; e < 8; ++e) lo[e] = fabsf(v[e]) < INFINITY ? lo[e] : (_Float16)0.f;
    to[0] = __builtin_bit_cast(f32x4, hi);
    if constexpr (HV == 2) to[4 * RM] = __builtin_bit_cast(f32x4, lo);
    return __builtin_amdgcn_ldexpf(1.f, 14 - e2);
  };
  // K blocks kb0 .. kb0 + nkb - 1 of the rows to LDS: 16 lanes take one of a
  // row, U of them at a time so that their loads are in flight together
  constexpr int U = RM <= 4 ? 1 : RM <= 16 ? 2 : 4, kTakers = W * 4;
  const XT* x = (const XT*)a.x + (int64_t)row0 * a.ld_x;
  float* units = (float*)(lds + sh.chunk * 16 * HV * RM);
  auto stage = [&](int kb0, int nkb) {
    const int dm = kTakers / nkb, dk = kTakers % nkb;
    for (int m = (tid >> 4) / nkb, kl = (tid >> 4) % nkb; m < rows;) {
      float v[U][8];
      int mu[U], ku[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (kb0 + kl) * kW4Rows + r16 * 8;
        load8(x + m * a.ld_x + k, m < rows ? a.K - k : 0, v[u]);
        mu[u] = m;
        ku[u] = kl;
        m += dm;
        kl += dk;
        if (kl >= nkb) {
          kl -= nkb;
          ++m;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (mu[u] >= rows) break;
        f32x4* to = lds + ((ku[u] * 4 + (r16 >> 2)) * HV * 4 + (r16 & 3)) * RM + (RM < 16 ? mu[u] : mu[u] ^ r16);
        const float unit = convert(v[u], to);
        if (r16 == 0) units[ku[u] * (16 * RT) + mu[u]] = unit;
      }
    }
  };

  const Masks masks;
  int x_row[4];  // where the lane's row of a step's fragments lies
#pragma unroll
  for (int s = 0; s < 4; ++s) x_row[s] = RM < 16 ? min(r16, RM - 1) : r16 ^ (4 * s + q);
  f32x4 sum[RT];
  auto compute = [&](const Block& b, int kl) {
    const f32x4* from = lds + (kl * 16 * HV + q) * RM;
    f32x4 acc[RT], part[RT], xf[2][RT][HV];
    auto fetch = [&](int s) {  // a step ahead of its products
#pragma unroll
      for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int z = 0; z < HV; ++z) xf[s & 1][i][z] = (from + x_row[s])[(s * HV + z) * 4 * RM + i * 16];
    };
    const uint32_t zeros4 = a.zeros ? (uint32_t)b.zero : 0x08080808u;
    fetch(0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      constexpr int kStepsPerGroup = 4 / GPB;
      const bool first = s % kStepsPerGroup == 0;
      const int g = s / kStepsPerGroup;
      if (s < 3) fetch(s + 1);
      // the group's zero point in both halves, and zl and zh as bits
      const uint32_t z = __builtin_amdgcn_perm(0u, zeros4, 0x0c000c00u | (uint32_t)g * 0x00010001u);
      const f16x2 zl = __builtin_bit_cast(f16x2, z | 0xac00ac00u);
      const f16x2 zh = __builtin_bit_cast(f16x2, (z << 4) | 0x9c009c00u);
      const uint32_t w = s == 0 ? b.code.x : s == 1 ? b.code.y : s == 2 ? b.code.z : b.code.w;
      const f16x8 c = codes_f16(w, zl, zh, masks);
#pragma unroll
      for (int h = HV - 1; h >= 0; --h)
#pragma unroll
        for (int i = 0; i < RT; ++i)
          acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, xf[s & 1][i][h]), c,
                                                          first && h == HV - 1 ? zero4() : acc[i], 0, 0, 0);
      if ((s + 1) % kStepsPerGroup == 0)
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            part[i][e] = g == 0 ? acc[i][e] * (float)b.scale[g] : fmaf(acc[i][e], (float)b.scale[g], part[i][e]);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
      const f32x4 unit = *(const f32x4*)(units + kl * (16 * RT) + i * 16 + 4 * q);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[i][e] = fmaf(part[i][e], unit[e], sum[i][e]);
    }
  };

  f32x4* red = lds + sh.chunk * (16 * HV * RM + 4 * RT) + wave * (RT * 64) + lane;
  // every wave goes round as often as the block's first has tiles
  for (int first = strip; first < a.tiles; first += tile_step, tile += tile_step) {
    const float bias = a.bias && tile < a.tiles ? a.bias[tile * kW4Cols + r16] : 0.f;
#pragma unroll
    for (int i = 0; i < RT; ++i) sum[i] = zero4();
    for (int kb0 = 0; kb0 < a.kblocks; kb0 += sh.chunk) {
      const int nkb = min(sh.chunk, a.kblocks - kb0);
      if (sh.chunk < a.kblocks || first < tile_step) {  // (all of K stays from the first time on)
        if (first >= tile_step || kb0 > 0) __syncthreads();
        stage(kb0, nkb);
        __syncthreads();
      }
      for (int j = 0; j < nkb; j += D * sh.wk) {
        // what comes after a slot's K block: one of these tiles, or of the next
        const bool more = kb0 + j + D * sh.wk < a.kblocks;
        const int next_tile = more ? tile : tile + tile_step, next_kb = more ? kb0 + j + D * sh.wk : 0;
#pragma unroll
        for (int d = 0; d < D; ++d) {
          const int kl = j + d * sh.wk + wk;
          if (kl < nkb && tile < a.tiles) compute(ring[d], kl);
          load(ring[d], next_tile, next_kb + d * sh.wk + wk);
        }
      }
    }
    if (sh.wk > 1) {  // the K shares' sums, in order
      if (first >= tile_step) __syncthreads();
      if (wk > 0)
#pragma unroll
        for (int i = 0; i < RT; ++i) red[i * 64] = sum[i];
      __syncthreads();
      if (wk > 0) continue;
      for (int w = 1; w < sh.wk; ++w)
#pragma unroll
        for (int i = 0; i < RT; ++i) sum[i] += red[(w * RT + i) * 64];
    }
    auto store = [&](auto* y) {
      using YT = std::remove_pointer_t<decltype(y)>;
      y += (row0 + 4 * q) * a.ld_y + (int64_t)tile * kW4Cols + r16;
      const int left = rows - 4 * q, cols = tile < a.tiles ? a.N - tile * kW4Cols - r16 : 0;
#pragma unroll
      for (int i = 0; i < RT; ++i, y += 12 * a.ld_y)
#pragma unroll
        for (int e = 0; e < 4; ++e, y += a.ld_y)
          if (i * 16 + e < left && cols > 0) *y = (YT)(sum[i][e] + bias);
    };
    if (a.y16)
      store((__bf16*)a.y);
    else
      store((float*)a.y);
  }
}

// Bytes of LDS that a K block takes.
constexpr int w4_block_bytes(int RM, bool x16) { return RM * (x16 ? 256 : 512) + (RM + 15) / 16 * 64; }

template <int RM, int W, int GPB, bool X16, bool S16>
hipError_t launch_form(const W4Args& a, const W4Shape& sh, hipStream_t st) {
  const int64_t grid = (int64_t)sh.strips * sh.row_blocks;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const size_t lds = (size_t)sh.chunk * w4_block_bytes(RM, X16) + (sh.wk > 1 ? (size_t)W * ((RM + 15) / 16) * 64 * 16 : 0);
  hipLaunchKernelGGL((k_w4_product<RM, W, GPB, X16, S16>), dim3((unsigned)grid), dim3(W * 64), lds, st, a, sh);
  return hipGetLastError();
}

hipError_t launch_product(const W4Args& a, bool x16, bool s16, int gpb, int cus, hipStream_t st) {
  // Row tiles a block: two, or three where those are all (48 rows of K = 500, N
  // = 100,000: 19.5 us in one block, 25 in two; more rows take as long either
  // way, and a fourth tile makes the waves spill), but only one while that
  // leaves fewer than eight waves a CU.
  W4Shape sh{};
  const int tiles16 = ceil_div(a.M, 16);
  auto groups_of = [&](int rt) { return (int64_t)a.tiles * ceil_div(tiles16, rt); };
  int RT = tiles16 <= 3 ? tiles16 : 2;
  while (RT > 1 && groups_of(RT) < 8 * cus) --RT;
  sh.row_blocks = ceil_div(tiles16, RT);
  RT = ceil_div(tiles16, sh.row_blocks);
  sh.rows = std::min(a.M, RT * 16);
  const int RM = a.M <= 4 ? 4 : RT * 16;
  // A K that half a CU's LDS does not hold gets all of it (less the K shares'
  // sums, which more than 16 rows never have): 5 rows of 4,000 x 1,000 in 24.0
  // us with half and 8 waves, 9.5 with all and 16, 16 rows 25.7 and 13.3.
  const int64_t bytes = w4_block_bytes(RM, x16);
  const bool long_k = a.kblocks * bytes > (56 << 10);
  const int W = w4_waves(RM, long_k), depth = w4_depth(RM, W, gpb), per_cu = W > 8 || long_k ? 1 : 2;
  const int most = std::max<int>(1, ((per_cu == 2 ? 56 : RM > 16 ? 160 : 144) << 10) / bytes);
  // K split between waves while there are fewer than about 8 waves a CU (a
  // block of several row tiles has them by itself)
  const int64_t groups = groups_of(RT);
  sh.wk = 1;
  while (sh.wk < W && groups * sh.wk < 8 * cus &&
         (most >= a.kblocks ? sh.wk * 2 <= a.kblocks : sh.wk * 2 * depth <= most))
    sh.wk *= 2;
  const int step = depth * sh.wk;
  sh.chunk = most >= a.kblocks ? a.kblocks : most / step * step;
  // as many blocks as run at once
  const int want = ceil_div(a.tiles, W / sh.wk), fit = per_cu * cus / sh.row_blocks;
  sh.strips = want <= fit ? (int)round_up(want, 8) : std::max(fit / 8 * 8, 8);
  auto types = [&](auto rm, auto w, auto g) {
    constexpr int R = decltype(rm)::value, V = decltype(w)::value, G = decltype(g)::value;
    return x16 ? (s16 ? launch_form<R, V, G, true, true>(a, sh, st) : launch_form<R, V, G, true, false>(a, sh, st))
               : (s16 ? launch_form<R, V, G, false, true>(a, sh, st) : launch_form<R, V, G, false, false>(a, sh, st));
  };
  auto form = [&](auto rm, auto w) {
    return gpb == 4   ? types(rm, w, std::integral_constant<int, 4>{})
           : gpb == 2 ? types(rm, w, std::integral_constant<int, 2>{})
                      : types(rm, w, std::integral_constant<int, 1>{});
  };
  using std::integral_constant;
  switch (RM) {
    case 4: return form(integral_constant<int, 4>{}, integral_constant<int, 8>{});
    case 16:
      return W == 8 ? form(integral_constant<int, 16>{}, integral_constant<int, 8>{})
                    : form(integral_constant<int, 16>{}, integral_constant<int, 16>{});
    case 32: return form(integral_constant<int, 32>{}, integral_constant<int, 16>{});
    default: return form(integral_constant<int, 48>{}, integral_constant<int, 16>{});
  }
}

bool known_type(int32_t t) { return t == NMT_F32 || t == NMT_BF16; }

// Checks the sizes and makes a matrix with its device memory; *out is only set
// on success.
nmt_status w4_new(const nmt_w4_dims& d, bool zeros, bool bias, nmt_w4** out) {
  if (d.K < 1 || d.N < 1) return entry_fail(NMT_EINVAL, "K and N must be positive");
  if (d.group < 32 || d.group % 32) return entry_fail(NMT_EINVAL, "group must be a positive multiple of 32");
  if (!known_type(d.stype)) return entry_fail(NMT_EINVAL, "unknown type of scales");
  nmt_w4* w = new (std::nothrow) nmt_w4();
  if (!w) return entry_fail(NMT_ENOMEM, "out of host memory");
  w->dims = d;
  w->tiles = ceil_div(d.N, kW4Cols);
  w->kblocks = ceil_div(d.K, kW4Rows);
  w->gpb = d.group % 128 == 0 ? 1 : d.group % 64 == 0 ? 2 : 4;
  hipError_t e = hipGetDevice(&w->device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&w->cus, hipDeviceAttributeMultiprocessorCount, w->device);
  size_t bytes = 0;
  auto part = [&](size_t n) {
    const size_t o = bytes;
    bytes += (n + 255) / 256 * 256;
    return o;
  };
  const size_t nsc = (size_t)w->tiles * w->kblocks * kW4Cols * w->gpb;
  const size_t o_codes = part((size_t)w->tiles * w->kblocks * 1024), o_sc = part(nsc * (d.stype == NMT_BF16 ? 2 : 4)),
               o_z = part(zeros ? nsc : 0), o_b = part(bias ? (size_t)w->tiles * kW4Cols * 4 : 0);
  if (e == hipSuccess) e = device_malloc(&w->mem, bytes);
  if (e != hipSuccess) {
    delete w;
    return entry_hip_fail(e, "4-bit matrix");
  }
  char* base = (char*)w->mem;
  w->codes = (uint4*)(base + o_codes);
  w->scales = base + o_sc;
  if (zeros) w->zeros = (uint8_t*)(base + o_z);
  if (bias) w->bias = (float*)(base + o_b);
  *out = w;
  return NMT_OK;
}

}  // namespace

extern "C" {

nmt_status nmt_w4_create(const nmt_w4_dims* dims, const uint8_t* h_codes, const float* h_scales,
                         const uint8_t* h_zeros, const float* h_bias, nmt_w4** out) {
  if (!out) return entry_fail(NMT_EINVAL, "NULL output");
  *out = nullptr;
  if (!dims || !h_codes || !h_scales) return entry_fail(NMT_EINVAL, "NULL argument");
  const nmt_w4_dims d = *dims;
  if (d.K < 1 || d.N < 1) return entry_fail(NMT_EINVAL, "K and N must be positive");
  if (d.group < 32 || d.group % 32) return entry_fail(NMT_EINVAL, "group must be a positive multiple of 32");
  if (!known_type(d.stype)) return entry_fail(NMT_EINVAL, "unknown type of scales");
  const size_t ng = (size_t)ceil_div(d.K, d.group) * d.N, nc = (size_t)d.K * (((size_t)d.N + 1) / 2);
  for (size_t i = 0; i < ng; ++i)
    if (!(std::fabs(h_scales[i]) <= kMostScale)) return entry_fail(NMT_EINVAL, "a scale is NaN or above 2^116");
  if (h_zeros)
    for (size_t i = 0; i < ng; ++i)
      if (h_zeros[i] > 15) return entry_fail(NMT_ERANGE, "a zero point is above 15");
  nmt_w4* w = nullptr;
  nmt_status rc = w4_new(d, h_zeros != nullptr, h_bias != nullptr, &w);
  if (rc != NMT_OK) return rc;
  // the host arrays as they are, laid out on the device
  auto al = [](size_t n) { return (n + 255) / 256 * 256; };
  const size_t o_s = al(nc), o_z = o_s + al(ng * 4), o_b = o_z + (h_zeros ? al(ng) : 0);
  char* raw = nullptr;
  hipError_t e = device_malloc((void**)&raw, o_b + (h_bias ? al((size_t)d.N * 4) : 0));
  if (e == hipSuccess) e = hipMemcpy(raw, h_codes, nc, hipMemcpyHostToDevice);
  if (e == hipSuccess) e = hipMemcpy(raw + o_s, h_scales, ng * 4, hipMemcpyHostToDevice);
  if (e == hipSuccess && h_zeros) e = hipMemcpy(raw + o_z, h_zeros, ng, hipMemcpyHostToDevice);
  if (e == hipSuccess && h_bias) e = hipMemcpy(raw + o_b, h_bias, (size_t)d.N * 4, hipMemcpyHostToDevice);
  if (e == hipSuccess) {
    const int64_t nv = (int64_t)w->tiles * w->kblocks * 64, np = (int64_t)w->tiles * w->kblocks * kW4Cols * w->gpb;
    hipLaunchKernelGGL(k_w4_pack, dim3((unsigned)((nv + 255) / 256)), dim3(256), 0, nullptr, (const uint8_t*)raw, d.K,
                       d.N, w->kblocks, nv, w->codes);
    auto params = [&](auto* s_out) {
      hipLaunchKernelGGL((k_w4_params<std::remove_pointer_t<decltype(s_out)>>), dim3((unsigned)((np + 255) / 256)),
                         dim3(256), 0, nullptr, (const float*)(raw + o_s),
                         h_zeros ? (const uint8_t*)(raw + o_z) : nullptr, h_bias ? (const float*)(raw + o_b) : nullptr,
                         d.K, d.N, d.group, w->kblocks, w->gpb, np, s_out, w->zeros, w->bias);
    };
    if (d.stype == NMT_BF16)
      params((__bf16*)w->scales);
    else
      params((float*)w->scales);
    e = hipGetLastError();
  }
  if (e == hipSuccess) e = hipDeviceSynchronize();
  device_free(raw);
  if (e != hipSuccess) {
    nmt_w4_destroy(w);
    return entry_hip_fail(e, "nmt_w4_create");
  }
  *out = w;
  return entry_ok();
}

nmt_status nmt_w4_from_output(const nmt_model* m, int32_t group, int32_t stype, void* stream, nmt_w4** out) {
  if (!out) return entry_fail(NMT_EINVAL, "NULL output");
  *out = nullptr;
  if (!m) return entry_fail(NMT_EINVAL, "NULL model");
  nmt_status rc = entry_check_device(m);
  if (rc != NMT_OK) return rc;
  const OutputLayer o = output_layer(m);
  nmt_w4* w = nullptr;
  rc = w4_new(nmt_w4_dims{o.E, o.V, group, stype}, false, true, &w);
  if (rc != NMT_OK) return rc;
  hipStream_t st = (hipStream_t)stream;
  const Packed& P = *o.W;
  const int64_t nv = (int64_t)w->tiles * w->kblocks * 64, np = (int64_t)w->tiles * w->kblocks * kW4Cols * w->gpb;
  int* bad = nullptr;
  int h_bad = 0;
  hipError_t e = device_malloc((void**)&bad, sizeof(int));
  if (e == hipSuccess) e = hipMemcpyAsync(bad, &h_bad, sizeof(int), hipMemcpyHostToDevice, st);
  auto quantise = [&](auto* sc) {
    using ST = std::remove_pointer_t<decltype(sc)>;
    hipLaunchKernelGGL((k_w4_out_scales<ST>), dim3((unsigned)((np + 255) / 256)), dim3(256), 0, st, P.d, (int)P.bf16,
                       P.Npad, o.E, o.V, group, w->kblocks, w->gpb, P.Krows, P.nbias, np, sc, w->bias, bad);
    hipLaunchKernelGGL((k_w4_out_codes<ST>), dim3((unsigned)((nv + 255) / 256)), dim3(256), 0, st, P.d, (int)P.bf16,
                       P.Npad, o.E, o.V, w->kblocks, w->gpb, nv, (const ST*)sc, w->codes);
  };
  if (e == hipSuccess) {
    if (stype == NMT_BF16)
      quantise((__bf16*)w->scales);
    else
      quantise((float*)w->scales);
    e = hipGetLastError();
  }
  if (e == hipSuccess) e = hipMemcpyAsync(&h_bad, bad, sizeof(int), hipMemcpyDeviceToHost, st);
  const hipError_t es = hipStreamSynchronize(st);
  if (e == hipSuccess) e = es;
  device_free(bad);
  if (e != hipSuccess || h_bad) {
    nmt_w4_destroy(w);
    return e != hipSuccess ? entry_hip_fail(e, "nmt_w4_from_output")
           : h_bad & 1     ? entry_fail(NMT_EINVAL, "the model's output layer has a weight that is not finite")
                           : entry_fail(NMT_EINVAL, "the model's output layer has a weight above 7 * 2^116");
  }
  *out = w;
  return entry_ok();
}

nmt_status nmt_w4_info(const nmt_w4* w, nmt_w4_dims* dims, int32_t* has_zeros, int32_t* has_bias) {
  if (!w) return entry_fail(NMT_EINVAL, "NULL matrix");
  if (dims) *dims = w->dims;
  if (has_zeros) *has_zeros = w->zeros != nullptr;
  if (has_bias) *has_bias = w->bias != nullptr;
  return entry_ok();
}

nmt_status nmt_w4_product(const nmt_w4* w, int32_t M, const void* d_x, int32_t x_type, int64_t ld_x, void* d_y,
                          int32_t y_type, int64_t ld_y, void* stream) {
  if (!w) return entry_fail(NMT_EINVAL, "NULL matrix");
  if (M < 0) return entry_fail(NMT_EINVAL, "M must be >= 0");
  if (!known_type(x_type) || !known_type(y_type)) return entry_fail(NMT_EINVAL, "unknown element type");
  if (M == 0) return entry_ok();
  if (!d_x || !d_y) return entry_fail(NMT_EINVAL, "a required device pointer is NULL");
  if (ld_x < w->dims.K || ld_y < w->dims.N) return entry_fail(NMT_EINVAL, "a row stride is below the row's length");
  const bool x16 = x_type == NMT_BF16, y16 = y_type == NMT_BF16;
  if (((uintptr_t)d_x & (x16 ? 1 : 3)) || ((uintptr_t)d_y & (y16 ? 1 : 3)))
    return entry_fail(NMT_EINVAL, "d_x and d_y must be aligned to their elements");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return entry_fail(NMT_EDEVICE, "hipGetDevice failed");
  if (dev != w->device) return entry_fail(NMT_EINVAL, "the 4-bit matrix lives on another device than the current one");
  constexpr int kMostRows = 1 << 20;  // of a launch, whose threads are counted in 32 bits
  for (int m0 = 0; m0 < M;) {
    const int n = std::min(M - m0, kMostRows);
    const W4Args a{w->codes, w->scales, w->zeros, w->bias, w->dims.K, w->dims.N, w->kblocks, w->tiles, n, y16,
                   (const char*)d_x + (int64_t)m0 * ld_x * (x16 ? 2 : 4), ld_x,
                   (char*)d_y + (int64_t)m0 * ld_y * (y16 ? 2 : 4), ld_y};
    const hipError_t e = launch_product(a, x16, w->dims.stype == NMT_BF16, w->gpb, w->cus, (hipStream_t)stream);
    if (e != hipSuccess) return entry_hip_fail(e, "nmt_w4_product");
    m0 += n;
  }
  return entry_ok();
}

void nmt_w4_destroy(nmt_w4* w) {
  if (!w) return;
  (void)hipDeviceSynchronize();
  device_free(w->mem);
  delete w;
}

}  // extern "C"
