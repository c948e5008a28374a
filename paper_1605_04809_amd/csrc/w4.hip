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
// zero points are kept per tile, [tile][group][16].
#include <cmath>
#include <new>

#include "draft.hpp"

using namespace nmt;

constexpr int kW4Cols = 16, kW4Rows = 128;  // columns and rows of a packed tile

struct nmt_w4 {
  nmt_w4_dims dims{};
  int device = 0, cus = 0;
  int tiles = 0, kblocks = 0, groups = 0;
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

// Scales (fp32 to ST, nearest even), zero points and bias into their places;
// zeros past the last column.
template <class ST>
__global__ __launch_bounds__(256) void k_w4_params(const float* __restrict__ scales, const uint8_t* __restrict__ zeros,
                                                   const float* __restrict__ bias, int N, int groups, int64_t n_all,
                                                   ST* __restrict__ s_out, uint8_t* __restrict__ z_out,
                                                   float* __restrict__ b_out) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_all) return;
  const int64_t tile = i / (kW4Cols * (int64_t)groups);
  const int g = (int)(i / kW4Cols % groups);
  const int64_t n = tile * kW4Cols + i % kW4Cols;
  s_out[i] = (ST)(n < N ? scales[(int64_t)g * N + n] : 0.f);
  if (zeros) z_out[i] = n < N ? zeros[(int64_t)g * N + n] : 0;
  if (bias && g == 0) b_out[n] = n < N ? bias[n] : 0.f;
}

// A model's output weight (k, n) from its packed matrix.
__device__ __forceinline__ float out_weight(const void* W, bool bf16, int64_t Npad, int k, int64_t n) {
  return bf16 ? (float)((const __bf16*)W)[((int64_t)(k / 8) * Npad + n) * 8 + k % 8]
              : ((const float*)W)[((int64_t)(k / 4) * Npad + n) * 4 + k % 4];
}

// Scales of the model's columns, one thread per (tile, group, column): the
// group's largest magnitude / 7.
template <class ST>
__global__ __launch_bounds__(256) void k_w4_out_scales(const void* __restrict__ W, int bf16, int64_t Npad, int K, int N,
                                                       int group, int groups, int krow, int nbias, int64_t n_all,
                                                       ST* __restrict__ s_out, float* __restrict__ b_out,
                                                       int* __restrict__ bad) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n_all) return;
  const int64_t tile = i / (kW4Cols * (int64_t)groups);
  const int g = (int)(i / kW4Cols % groups);
  const int64_t n = tile * kW4Cols + i % kW4Cols;
  float mx = 0.f;
  bool finite = true;
  if (n < N) {
    const int k1 = min(K, (g + 1) * group);
    for (int k = g * group; k < k1; ++k) {
      const float a = fabsf(out_weight(W, bf16, Npad, k, n));
      finite = finite && a < INFINITY;
      mx = fmaxf(mx, a);
    }
    if (g == 0) {
      float b = 0.f;
      for (int j = 0; j < nbias; ++j) b += out_weight(W, bf16, Npad, krow + j, n);
      b_out[n] = b;
    }
  } else if (g == 0) {
    b_out[n] = 0.f;
  }
  s_out[i] = (ST)(mx / 7.f);
  // (a scale that rounds up to infinity is as useless as an infinite weight)
  if (!finite || !((float)(ST)(mx / 7.f) < INFINITY)) atomicOr(bad, 1);
}

// The codes under those scales, one packed vector per thread.
template <class ST>
__global__ __launch_bounds__(256) void k_w4_out_codes(const void* __restrict__ W, int bf16, int64_t Npad, int K, int N,
                                                      int group, int groups, int kblocks, int64_t n_all,
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
        const float sc = (float)scales[(tile * groups + k / group) * kW4Cols + r];
        const float v = sc != 0.f ? rintf(out_weight(W, bf16, Npad, k, n) / sc) : 0.f;
        c = (uint32_t)(8 + (int)fminf(fmaxf(v, -7.f), 7.f));
      }
      w[s] |= c << (4 * p);
    }
  }
  out[i] = uint4{w[0], w[1], w[2], w[3]};
}

// ------------------------------------------------------------- product

struct W4Args {
  const uint4* codes;
  const void* scales;
  const uint8_t* zeros;
  const float* bias;
  int K, N, group, groups, kblocks, M;
  const void* x;
  int64_t ld_x;
  void* y;
  int64_t ld_y;
};

// One output a thread: 16 columns of a tile times 16 rows of x in a block.
template <class XT, class YT, class ST>
__global__ __launch_bounds__(256) void k_w4_product(W4Args a) {
  const int r = threadIdx.x & 15;
  const int64_t tile = blockIdx.x, n = tile * kW4Cols + r, m = (int64_t)blockIdx.y * 16 + (threadIdx.x >> 4);
  if (n >= a.N || m >= a.M) return;
  const XT* x = (const XT*)a.x + m * a.ld_x;
  float sum = 0.f, part = 0.f;
  for (int k0 = 0; k0 < a.K; k0 += 8) {
    const int s = k0 / 32 % 4, q = k0 / 8 % 4, g = k0 / a.group;
    const uint32_t w = ((const uint32_t*)(a.codes + (tile * a.kblocks + k0 / kW4Rows) * 64 + q * 16 + r))[s];
    const float z = a.zeros ? (float)a.zeros[(tile * a.groups + g) * kW4Cols + r] : 8.f;
    for (int p = 0; p < 8; ++p) {
      const int k = k0 + nibble_row(p);
      if (k < a.K) part = fmaf((float)x[k], (float)((w >> (4 * p)) & 15u) - z, part);
    }
    if ((k0 + 8) % a.group == 0 || k0 + 8 >= a.K) {
      sum = fmaf(part, (float)((const ST*)a.scales)[(tile * a.groups + g) * kW4Cols + r], sum);
      part = 0.f;
    }
  }
  if (a.bias) sum += a.bias[n];
  ((YT*)a.y)[m * a.ld_y + n] = (YT)sum;
}

template <class XT, class YT, class ST>
hipError_t launch_product(const W4Args& a, int tiles, hipStream_t st) {
  for (int m0 = 0; m0 < a.M; m0 += 16 * 65535) {  // rows per launch: the grid's limit
    W4Args b = a;
    b.M = a.M - m0 < 16 * 65535 ? a.M - m0 : 16 * 65535;
    b.x = (const XT*)a.x + (int64_t)m0 * a.ld_x;
    b.y = (YT*)a.y + (int64_t)m0 * a.ld_y;
    hipLaunchKernelGGL((k_w4_product<XT, YT, ST>), dim3(tiles, ceil_div(b.M, 16)), dim3(256), 0, st, b);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
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
  w->groups = ceil_div(d.K, d.group);
  hipError_t e = hipGetDevice(&w->device);
  if (e == hipSuccess) e = hipDeviceGetAttribute(&w->cus, hipDeviceAttributeMultiprocessorCount, w->device);
  size_t bytes = 0;
  auto part = [&](size_t n) {
    const size_t o = bytes;
    bytes += (n + 255) / 256 * 256;
    return o;
  };
  const size_t nsc = (size_t)w->tiles * w->groups * kW4Cols;
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
  // the largest fp32 below what rounds to a bf16 infinity
  const float most = d.stype == NMT_BF16 ? 0x1.fefffep127f : 0x1.fffffep127f;
  for (size_t i = 0; i < ng; ++i)
    if (!(std::fabs(h_scales[i]) <= most)) return entry_fail(NMT_EINVAL, "a scale is not finite in the scales' type");
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
    const int64_t nv = (int64_t)w->tiles * w->kblocks * 64, np = (int64_t)w->tiles * w->groups * kW4Cols;
    hipLaunchKernelGGL(k_w4_pack, dim3((unsigned)((nv + 255) / 256)), dim3(256), 0, nullptr, (const uint8_t*)raw, d.K,
                       d.N, w->kblocks, nv, w->codes);
    auto params = [&](auto* s_out) {
      hipLaunchKernelGGL((k_w4_params<std::remove_pointer_t<decltype(s_out)>>), dim3((unsigned)((np + 255) / 256)),
                         dim3(256), 0, nullptr, (const float*)(raw + o_s),
                         h_zeros ? (const uint8_t*)(raw + o_z) : nullptr, h_bias ? (const float*)(raw + o_b) : nullptr,
                         d.N, w->groups, np, s_out, w->zeros, w->bias);
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
  const int64_t nv = (int64_t)w->tiles * w->kblocks * 64, np = (int64_t)w->tiles * w->groups * kW4Cols;
  int* bad = nullptr;
  int h_bad = 0;
  hipError_t e = device_malloc((void**)&bad, sizeof(int));
  if (e == hipSuccess) e = hipMemcpyAsync(bad, &h_bad, sizeof(int), hipMemcpyHostToDevice, st);
  auto quantise = [&](auto* sc) {
    using ST = std::remove_pointer_t<decltype(sc)>;
    hipLaunchKernelGGL((k_w4_out_scales<ST>), dim3((unsigned)((np + 255) / 256)), dim3(256), 0, st, P.d, (int)P.bf16,
                       P.Npad, o.E, o.V, group, w->groups, P.Krows, P.nbias, np, sc, w->bias, bad);
    hipLaunchKernelGGL((k_w4_out_codes<ST>), dim3((unsigned)((nv + 255) / 256)), dim3(256), 0, st, P.d, (int)P.bf16,
                       P.Npad, o.E, o.V, group, w->groups, w->kblocks, nv, (const ST*)sc, w->codes);
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
                           : entry_fail(NMT_EINVAL, "the model's output layer has a weight that is not finite");
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
  const bool x16 = x_type == NMT_BF16, y16 = y_type == NMT_BF16, s16 = w->dims.stype == NMT_BF16;
  if (((uintptr_t)d_x & (x16 ? 1 : 3)) || ((uintptr_t)d_y & (y16 ? 1 : 3)))
    return entry_fail(NMT_EINVAL, "d_x and d_y must be aligned to their elements");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) return entry_fail(NMT_EDEVICE, "hipGetDevice failed");
  if (dev != w->device) return entry_fail(NMT_EINVAL, "the 4-bit matrix lives on another device than the current one");
  const W4Args a{w->codes, w->scales, w->zeros, w->bias, w->dims.K, w->dims.N, w->dims.group, w->groups, w->kblocks, M,
                 d_x, ld_x, d_y, ld_y};
  hipStream_t st = (hipStream_t)stream;
  auto scales = [&](auto xt, auto yt) {
    return s16 ? launch_product<decltype(xt), decltype(yt), __bf16>(a, w->tiles, st)
               : launch_product<decltype(xt), decltype(yt), float>(a, w->tiles, st);
  };
  const hipError_t e = x16 ? (y16 ? scales(__bf16{}, __bf16{}) : scales(__bf16{}, float{}))
                           : (y16 ? scales(float{}, __bf16{}) : scales(float{}, float{}));
  if (e != hipSuccess) return entry_hip_fail(e, "nmt_w4_product");
  return entry_ok();
}

void nmt_w4_destroy(nmt_w4* w) {
  if (!w) return;
  (void)hipDeviceSynchronize();
  device_free(w->mem);
  delete w;
}

}  // extern "C"
