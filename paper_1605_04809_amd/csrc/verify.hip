// verify.hip -- which drafted words a model's distributions keep, and the word
// after them (nmt_verify_drafts).
//
// With p_j the target's softmax at position j and q_j the one that draft d_j
// was drawn from, draft j is kept with probability min(1, p_j(d_j) / q_j(d_j))
// (u_j q_j(d_j) < p_j(d_j) for a uniform u_j), and the first one that is not
// is replaced by a word drawn from max(p_j - q_j, 0): the word at position j
// is v with probability min(p(v), q(v)) + (1 - sum_w min(p(w), q(w))) times
// max(p(v) - q(v), 0) / sum_w max(p(w) - q(w), 0), which is p(v).
//
// The results are whole numbers decided by comparisons, so everything behind a
// comparison is in 64 bits: each row's sum of exponentials, the residual's
// running sum.  The exponentials themselves are right to 1e-10 of themselves
// (exp64 and add_exp say why that does).
//
// As a rule there are two launches.  k_row_sums reads every row once: a wave
// takes up to 2,048 logits into registers, all loads in flight at once, and a
// block leaves the (max, sum) pair of up to 8,192.  fp32 rows keep it at the
// rate of memory (79 M logits, 317 MB, in 50 us), bf16 ones at that of its
// 64-bit instructions (30 M logits in 22.5 us, 15 of them VALU; parts half or
// twice as long: 1 and 3 us more).  k_finish judges its sequence from those
// pairs (each block by itself: 16 lanes merge a row, then a lane decides a
// position), sums what is left of the target over its share of the words, 512
// at a time, and the sequence's last block to finish finds the 512, then the
// word, whose running sum passes the random number.  It is a chain of some
// eight dependent trips to memory (9 to 10 us for 12 sequences, three quarters
// of its waves' time) until the rows themselves count (256 sequences of 100,000
// words: 102 MB in 32 us).  Both stages are spread over the whole chip, so one
// sequence takes no longer than its share of the bandwidth; every sum has a
// fixed order.  Few sequences over a small vocabulary take one launch, a block
// a sequence (k_verify_small).
#include <algorithm>

#include "draft.hpp"

using namespace nmt;

namespace {

constexpr int kWavePart = 2048;   // logits of a row that one wave sums, at most
constexpr int kWaves = 4;         // waves a block of the streaming kernels
constexpr int kUnit = 512;        // words whose residual one wave sums at a time
constexpr int kFinish = 8;        // waves a block that judges long rows ...
constexpr int kJudge = 16;        // ... and positions it judges at a time, 16 lanes a row
constexpr int kSmall = 8;         // positions that a block of the one-launch form judges at a time

// A row's (or a part's) largest logit and the sum of e^(z - max).  A NaN makes
// the max NaN, and a row of nothing but -infinity has max -infinity and sum 0.
struct RowSum {
  double s;
  float m;
};
__device__ __forceinline__ bool is_distribution(const RowSum& r) {
  return r.m > -INFINITY && r.m < INFINITY && r.s > 0.0 && r.s < INFINITY;
}

// Where a sequence's words come to an end.
struct Verdict {
  int64_t t_row, p_row;  // the rows that the next word is drawn from (p_row -1: the target's alone)
  double it, ip;         // one over their sums
  float mt, mp;
  int32_t kept, bad;     // bad: no word follows (and which bits of the error flag)
  int32_t cut;           // without proposals: the word that p goes without (-1: none)
  int32_t whole;         // the residual holds nothing: p itself
};

struct VerifyArgs {
  int S, n_draft, V;
  int parts, part_len, units;     // parts of a row and their length, units of a residual
  const int32_t *off, *draft;
  const void *target, *proposal;  // proposal null: drafts are certain
  int target16, proposal16;
  int64_t ld_t, ld_p;
  const float* u;
  int32_t *accepted, *next;
  float *draft_logp, *next_logp;  // nullable
  // workspace: parts of the target's rows, then the proposal's; units of the
  // sequences' residuals; blocks of a sequence that have finished
  RowSum* rows;
  double* rest;
  uint32_t* done;
  int* err;
};

__device__ __forceinline__ float logit(const void* z, int is16, int64_t i) {
  return is16 ? (float)((const __bf16*)z)[i] : ((const float*)z)[i];
}

// e^x as 2^n e^r, |r| <= ln 2 / 2, e^r by the polynomial that interpolates it
// at the Chebyshev nodes (off by at most 5.6e-11 of it, and exact at 0), in 11
// 64-bit instructions.  The odds that an error of the sums (at most 1e-10 of
// them, from add_exp below) moves a decision are its part of the distance
// between two borders: 1e-10 for a draft, and 1e-5 for a word out of 100,000
// equal ones even if every error had the same sign.
__device__ __forceinline__ double exp64(double x) {
  constexpr double kShift = 6755399441055744.0;  // 1.5 * 2^52: n comes out in the sum's low bits
  const double t = fma(x, 1.4426950408889634, kShift);
  const double r = fma(t - kShift, -0.6931471805599453, x);
  double p = 0.00019907567086439808;
  p = fma(p, r, 0.0013948578255139586);
  p = fma(p, r, 0.00833328354312129);
  p = fma(p, r, 0.04166621832056651);
  p = fma(p, r, 0.16666666786284912);
  p = fma(p, r, 0.5000000107728596);
  p = fma(p, r, 0.9999999999955115);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)(uint32_t)__builtin_bit_cast(uint64_t, t));
}
constexpr double kNothing = -760.0;  // e^-760 is 0
__device__ __forceinline__ double exp_rel(float z, float m) { return exp64(fmax((double)z - (double)m, kNothing)); }

// ------------------------------------------------------- lane arithmetic

__device__ __forceinline__ int wave_index() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// v of the lane that `ctrl` names (0 where there is none).
template <int kCtrl, int kRows = 0xf>
__device__ __forceinline__ double dpp(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, kCtrl, kRows, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), kCtrl, kRows, 0xf, false);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, false));
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kMirror8 = 0x141, kMirror16 = 0x140;  // within 4, 4, 8, 16 lanes

// Running sums over the wave's lanes, each lane's own included.
__device__ __forceinline__ double wave_scan(double v) {
  v += dpp<0x111>(v);  // the lane 1, 2, 4, 8 before, within 16
  v += dpp<0x112>(v);
  v += dpp<0x114>(v);
  v += dpp<0x118>(v);
  v += dpp<0x142, 0xa>(v);  // the last of the 16 before, to every second 16
  v += dpp<0x143, 0xc>(v);  // the last of the first 32, to the others
  return v;
}
__device__ __forceinline__ double lane_value(double v, int lane) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = __builtin_amdgcn_readlane((int)(uint32_t)b, lane);
  const uint32_t hi = __builtin_amdgcn_readlane((int)(uint32_t)(b >> 32), lane);
  return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
__device__ __forceinline__ double wave_sum(double v) { return lane_value(wave_scan(v), 63); }
// The lane before's (0 in the first).
__device__ __forceinline__ double lane_before(double v) { return dpp<0x138>(v); }

// maximum() returns NaN if either is (fmaxf does not).
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float maximum16(float v) {  // of 16 lanes, in all of them
  v = maximum(v, dpp<kXor1>(v));
  v = maximum(v, dpp<kXor2>(v));
  v = maximum(v, dpp<kMirror8>(v));
  return maximum(v, dpp<kMirror16>(v));
}
__device__ __forceinline__ double sum16(double v) {
  v += dpp<kXor1>(v);
  v += dpp<kXor2>(v);
  v += dpp<kMirror8>(v);
  return v + dpp<kMirror16>(v);
}
__device__ __forceinline__ float wave_maximum(float v) {
  v = maximum16(v);
  v = maximum(v, __shfl_xor(v, 16, 64));
  return maximum(v, __shfl_xor(v, 32, 64));
}

// Eight consecutive logits of the row at z[row], from w0, or where those would
// pass V the row's last eight; any alignment of the elements' own.  They come
// as they are in memory (bf16 ones in x[0 .. 3]), so that nothing waits for
// them before ready8, which makes floats of them, -infinity for those before
// w0.  Returns where they start.  With kShort rows of less than eight words are
// met, of which a lane has one: each_lane() words a lane.  (The type is a branch
// here, the same for the whole wave, and not a form of each kernel: their code
// would double, and a block that runs once waits for its instructions as for
// its data.)
typedef float f32x8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ int each_lane(int V) { return V < 8 ? 1 : 8; }
template <bool kShort>
__device__ __forceinline__ int load8(const void* z, int is16, int64_t row, int w0, int V, f32x8& x) {
  if (kShort && V < 8) {
    x = is16 ? as_float(0xff80ff80u) : -INFINITY;
    if (is16)
      x[0] = as_float(0xff800000u | (w0 < V ? ((const uint16_t*)z)[row + w0] : 0xff80u));
    else
      x[0] = w0 < V ? ((const float*)z)[row + w0] : -INFINITY;
    return w0;
  }
  const int at = min(w0, V - 8);
  if (is16) {
    typedef float f32x4h __attribute__((ext_vector_type(4), aligned(2)));
    const f32x4h a = *(const f32x4h*)((const uint16_t*)z + row + at);
    x = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
  } else {
    const f32x4u* p = (const f32x4u*)((const float*)z + row + at);
    const f32x4u a = p[0], b = p[1];
    x = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  return at;
}
__device__ __forceinline__ void ready8(int is16, int at, int w0, f32x8& x) {
  if (is16) {
    f32x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t u = __float_as_uint(x[e / 2]);
      y[e] = as_float(e & 1 ? u & 0xffff0000u : u << 16);
    }
    x = y;
  }
  if (at < w0) {
    f32x8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = at + e < w0 ? -INFINITY : x[e];
    x = y;
  }
}

// ------------------------------------------------------------- row sums

// 2^(j / 32) as a double's bits, less j << 15 in the upper half: n << 15 on
// that puts n / 32 on the exponent, whole steps alone.  (Exponentials from a
// table of 2^(j / 32) are P. T. P. Tang's, ACM TOMS 15(2), 1989; the polynomials
// here interpolate at Chebyshev nodes.)
__device__ const uint64_t kPowers[32] = {
    0x3ff0000000000000, 0x3fefd9b0d3158574, 0x3fefb5586cf9890f, 0x3fef9301d0125b51,
    0x3fef72b83c7d517b, 0x3fef54873168b9aa, 0x3fef387a6e756238, 0x3fef1e9df51fdee1,
    0x3fef06fe0a31b715, 0x3feef1a7373aa9cb, 0x3feedea64c123422, 0x3feece086061892d,
    0x3feebfdad5362a27, 0x3feeb42b569d4f82, 0x3feeab07dd485429, 0x3feea47eb03a5585,
    0x3feea09e667f3bcd, 0x3fee9f75e8ec5f74, 0x3feea11473eb0187, 0x3feea589994cce13,
    0x3feeace5422aa0db, 0x3feeb737b0cdc5e5, 0x3feec49182a3f090, 0x3feed503b23e255d,
    0x3feee89f995ad3ad, 0x3feeff76f2fb5e47, 0x3fef199bdd85529c, 0x3fef3720dcef9069,
    0x3fef5818dcfba487, 0x3fef7c97337b9b5f, 0x3fefa4afa2a490da, 0x3fefd0765b6e4540,
};
// sum + e^x for x from -700 to 700: as exp64, but in steps of ln 2 / 32, so
// that a polynomial of degree 3 does (off by at most 9.9e-11 of e^x), times a
// factor from the table: 8 64-bit instructions with the addition, and 4 of 32
// bits (row sums of 64 sequences: 28.5 us with exp64).  The table's 32 doubles
// fill the 64 banks once, so lanes never wait for each other.
constexpr float kLowest = -700.f;
__device__ __forceinline__ double add_exp(double sum, float x, const uint64_t* table) {
  constexpr double kShift = 6755399441055744.0;
  const double d = maximum(x, kLowest);
  const double t = fma(d, 46.16624130844683, kShift);
  const double r = fma(t - kShift, -0.02166084939249829, d);
  const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
  const uint64_t b = table[n & 31];
  uint32_t hi;  // (the compiler would take a 64-bit addition for it)
  asm("v_lshl_add_u32 %0, %1, 15, %2" : "=v"(hi) : "v"(n), "v"((uint32_t)(b >> 32)));
  const double p = fma(fma(fma(0.16666804903930896, r, 0.5000040488943809), r, 0.9999999999525067), r, 1.0);
  return fma(__builtin_bit_cast(double, (uint64_t)hi << 32 | (uint32_t)b), p, sum);
}

// Up to kWavePart logits of a row, from word `from` to `to` or the row's end,
// on their way to one wave, and their pair.  A largest of ordinary size is not
// taken off each logit but divided out of their sum: its own term still counts
// exactly 1.
constexpr float kPlain = 200.f;  // 2,048 e^200 and e^-200 are far inside a double's range
constexpr int kSteps = kWavePart / 512;  // eight logits a lane and step
template <bool kShort>
struct Part {
  const void* z;
  int is16, from, to, V, w0;
  int64_t row;
  f32x8 x[kSteps];
  int at[kSteps];

  __device__ __forceinline__ Part(const void* z, int is16, int64_t row, int from, int to, int V)
      : z(z), is16(is16), from(from), to(min(to, V)), V(V),
        w0(from + (int)(threadIdx.x & 63) * (kShort ? each_lane(V) : 8)), row(row) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i)
      if (this->from + i * 512 < this->to) at[i] = load8<kShort>(z, is16, row, w0 + i * 512, V, x[i]);
  }

  __device__ __forceinline__ RowSum sum(const uint64_t* table) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (from + i * 512 >= to) break;  // (a short part has few steps)
      ready8(is16, at[i], w0 + i * 512, x[i]);
#pragma unroll
      for (int e = 0; e < 8; ++e) m = maximum(m, x[i][e]);
    }
    m = wave_maximum(m);
    double s = 0.0;
    if (m >= -kPlain && m <= kPlain) {
      double s1 = 0.0;
#pragma unroll
      for (int i = 0; i < kSteps; ++i) {
        if (from + i * 512 >= to) break;
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          s = add_exp(s, x[i][e], table);
          s1 = add_exp(s1, x[i][e + 1], table);
        }
      }
      s = wave_sum(s + s1) / add_exp(0.0, m, table);
    } else if (m > -INFINITY && m < INFINITY) {
#pragma unroll 1
      for (int i = 0; from + i < to; i += 512) {
        ready8(is16, load8<kShort>(z, is16, row, w0 + i, V, x[0]), w0 + i, x[0]);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += exp_rel(x[0][e], m);
      }
      s = wave_sum(s);
    }
    return RowSum{s, m};
  }
};

__device__ __forceinline__ RowSum merge(const RowSum& a, const RowSum& b) {
  const float m = maximum(a.m, b.m);
  if (!(m > -INFINITY && m < INFINITY)) return RowSum{0.0, m};
  return RowSum{a.s * exp_rel(a.m, m) + b.s * exp_rel(b.m, m), m};
}

// One block per part of a row.
__global__ __launch_bounds__(kWaves * 64) void k_row_sums(VerifyArgs a) {
  __shared__ RowSum sums[kWaves];
  __shared__ uint64_t table[32];
  const int64_t row = blockIdx.x / a.parts;
  const int part = blockIdx.x % a.parts, wave = wave_index();
  const int64_t thread = (int64_t)blockIdx.x * (kWaves * 64) + threadIdx.x;
  if (thread < a.S) a.done[thread] = 0;  // (as many threads as sequences at least)
  const int64_t n_target = (int64_t)a.n_draft + a.S;
  const bool tgt = row < n_target;
  const int from = part * a.part_len + wave * (a.part_len / kWaves);
  const uint64_t power = kPowers[threadIdx.x & 31];  // (before the logits, or it waits for them)
  Part<false> part_of(tgt ? a.target : a.proposal, tgt ? a.target16 : a.proposal16,
                      tgt ? row * a.ld_t : (row - n_target) * a.ld_p, from, from + a.part_len / kWaves, a.V);
  if (threadIdx.x < 32) table[threadIdx.x] = power;
  __syncthreads();
  const RowSum r = part_of.sum(table);
  if ((threadIdx.x & 63) == 0) sums[wave] = r;
  __syncthreads();
  if (threadIdx.x == 0) a.rows[blockIdx.x] = merge(merge(sums[0], sums[1]), merge(sums[2], sums[3]));
}

// --------------------------------------------------------------- verdict

// The verdict on sequence s by one block, J positions at a time: fill(j0,
// rows) leaves the sums of their target rows and proposal rows, then the first
// wave takes a lane a position.  With write_logp log p of each draft goes out
// too, and every position is looked at for it.  *out holds the verdict after
// the call, for the whole block.
template <int J, class Fill>
__device__ __forceinline__ void judge(const VerifyArgs& a, int s, int o0, int o1, bool write_logp, Verdict* out,
                                      Fill&& fill) {
  __shared__ RowSum rows[2][J];
  __shared__ int done;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (o0 < 0 || o1 < o0 || o1 > a.n_draft) {
    if (threadIdx.x == 0) {
      *out = Verdict{};
      out->bad = 1;
    }
    __syncthreads();
    return;
  }
  const int n = o1 - o0;
  if (threadIdx.x == 0) done = 0;
  for (int j0 = 0; j0 <= n; j0 += J) {
    // what else a position is judged by, on its way while the sums are made
    const int j = j0 + lane;
    const bool pos = wave == 0 && lane < J && j <= n, has_p = pos && j < n && a.proposal;
    const int64_t tr = (int64_t)o0 + s + j, pr = (int64_t)o0 + j;
    const int32_t d = pos && j < n ? a.draft[pr] : 0;
    const float u = pos ? a.u[tr] : 0.f;
    const bool d_ok = d >= 0 && d < a.V;
    const float zt = pos ? logit(a.target, a.target16, tr * a.ld_t + (d_ok ? d : 0)) : 0.f;
    const float zp = has_p ? logit(a.proposal, a.proposal16, pr * a.ld_p + (d_ok ? d : 0)) : 0.f;
    fill(j0, n, rows);
    __syncthreads();
    if (wave == 0) {
      const RowSum rt = rows[0][lane % J], rp = has_p ? rows[1][lane % J] : RowSum{1.0, 0.f};
      const bool t_ok = is_distribution(rt);
      const int bad = !d_ok ? 1 : !t_ok || !is_distribution(rp) ? 2 : 0;
      const double it = 1.0 / rt.s, ip = 1.0 / rp.s;
      const double p = exp_rel(zt, rt.m) * it;
      const double q = has_p ? exp_rel(zp, rp.m) * ip : 1.0;
      const bool end = pos && (j == n || bad || !((double)u * q < p));
      const uint64_t ends = __ballot(end);
      if (!done && ends && lane == __builtin_ctzll(ends)) {
        *out = Verdict{tr, has_p ? pr : -1, it, ip, rt.m, rp.m, j, bad, j < n && !a.proposal ? d : -1, 0};
        done = 1;
      }
      if (write_logp && pos && j < n)
        a.draft_logp[pr] = d_ok && t_ok ? (float)((double)zt - (double)rt.m - log(rt.s)) : __builtin_nanf("");
    }
    __syncthreads();
    if (done && !write_logp) break;
  }
}

// A sequence that no word follows.
__device__ __forceinline__ void write_bad(const VerifyArgs& a, int s, const Verdict& v) {
  a.accepted[s] = v.kept;
  a.next[s] = -1;
  if (a.next_logp) a.next_logp[s] = __builtin_nanf("");
  atomicOr(a.err, v.bad);
}

// -------------------------------------------------------------- residual

// What is left of eight words for the draw: those from w0, or the last eight,
// in which those before w0 count nothing.  `at` is where they start.
struct Logits8 {
  f32x8 t, p;
  int at;
};
__device__ __forceinline__ bool minus_proposal(const Verdict& v) { return v.p_row >= 0 && !v.whole; }
template <bool kShort>
__device__ __forceinline__ void load_residual8(const VerifyArgs& a, const Verdict& v, int w0, Logits8& x) {
  x.at = load8<kShort>(a.target, a.target16, v.t_row * a.ld_t, w0, a.V, x.t);
  if (minus_proposal(v)) load8<kShort>(a.proposal, a.proposal16, v.p_row * a.ld_p, w0, a.V, x.p);
}
__device__ __forceinline__ void residual8(const VerifyArgs& a, const Verdict& v, int w0, Logits8& x, double (&r)[8]) {
  ready8(a.target16, x.at, w0, x.t);
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = exp_rel(x.t[e], v.mt) * v.it;
  if (minus_proposal(v)) {
    // (both products rounded, and not one inside a multiply-add: equal rows leave nothing)
#pragma clang fp contract(off)
    ready8(a.proposal16, x.at, w0, x.p);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const double q = exp_rel(x.p[e], v.mp) * v.ip;
      r[e] = fmax(r[e] - q, 0.0);
    }
  } else if (v.cut >= 0 && !v.whole) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = x.at + e == v.cut ? 0.0 : r[e];
  }
}
__device__ __forceinline__ double sum8(const double (&r)[8]) {
  return ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
}

// The first of a lane's words (eight from `at`, residuals r, running sum before
// them `run`) whose running sum passes the goal, and the last that has any.
struct Picked {
  int hit, last;
};
constexpr int kNone = 0x7fffffff;
__device__ __forceinline__ Picked pick8(const double (&r)[8], double run, double goal, int at) {
  Picked p{kNone, -1};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    run += r[e];
    if (r[e] > 0.0) {
      if (run > goal && p.hit == kNone) p.hit = at + e;
      p.last = at + e;
    }
  }
  return p;
}
// The wave's.
__device__ __forceinline__ Picked pick_wave(Picked p) {
  const uint64_t hit = __ballot(p.hit != kNone), any = __ballot(p.last >= 0);
  return Picked{hit ? __builtin_amdgcn_readlane(p.hit, __builtin_ctzll(hit)) : kNone,
                any ? __builtin_amdgcn_readlane(p.last, 63 - __builtin_clzll(any)) : -1};
}

__device__ __forceinline__ void write_next(const VerifyArgs& a, int s, const Verdict& v, int w) {
  a.accepted[s] = v.kept;
  a.next[s] = w;
  if (a.next_logp)
    a.next_logp[s] = (float)((double)logit(a.target, a.target16, v.t_row * a.ld_t + w) - (double)v.mt + log(v.it));
}

// `blocks` blocks a sequence: the verdict, the residual over every blocks-th
// 2,048 words, and by the last to finish the word.
__global__ __launch_bounds__(kFinish * 64) void k_finish(VerifyArgs a, int blocks) {
  __shared__ Verdict shared_v;
  __shared__ int last_block;
  const int s = blockIdx.x / blocks, b = blockIdx.x % blocks, lane = threadIdx.x & 63, wave = wave_index();
  const int o0 = a.off[s], o1 = a.off[s + 1];
  const float u = o1 >= 0 && o1 <= a.n_draft ? a.u[(int64_t)o1 + s] : 0.f;
  judge<kJudge>(a, s, o0, o1, b == 0 && a.draft_logp, &shared_v, [&](int j0, int n, RowSum(&rows)[2][kJudge]) {
    const int g = threadIdx.x >> 4, l16 = threadIdx.x & 15, j = j0 + g % kJudge;
    const bool prop = g >= kJudge;
    RowSum mine{0.0, -INFINITY};
    if (j < n + (prop ? 0 : 1) && (!prop || a.proposal)) {
      const int64_t row = prop ? (int64_t)a.n_draft + a.S + o0 + j : (int64_t)o0 + s + j;
      for (int i = l16; i < a.parts; i += 16) {
        const RowSum p = a.rows[row * a.parts + i];
        mine = i < 16 ? p : merge(mine, p);
      }
    }
    const float m = maximum16(mine.m);
    const bool ok = m > -INFINITY && m < INFINITY;
    const double sum = sum16(ok ? mine.s * exp_rel(mine.m, m) : 0.0);
    if (l16 == 0) rows[prop][g % kJudge] = RowSum{sum, m};
  });
  Verdict v = shared_v;
  if (v.bad) {
    if (b == 0 && threadIdx.x == 0) write_bad(a, s, v);
    return;
  }
  double* rest = a.rest + (int64_t)s * a.units;
  // units first, first + step, ..., the next one's logits on their way
  auto sum_units = [&](int first, int step) {
    Logits8 x, next;
    for (int i = first, now = -1;; now = i, i += step, x = next) {
      if (i < a.units) load_residual8<false>(a, v, i * kUnit + lane * 8, next);
      if (now >= 0) {
        double r[8];
        residual8(a, v, now * kUnit + lane * 8, x, r);
        const double sum = wave_sum(sum8(r));
        if (lane == 0) __hip_atomic_store(rest + now, sum, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      if (i >= a.units) break;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  };
  // four consecutive units a lane; each(the first, their sums, the sum before them); returns the whole sum
  auto running = [&](auto&& each) {
    double sum = 0.0;
    for (int i0 = 0; i0 < a.units; i0 += 256) {
      double x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = i0 + lane * 4 + e < a.units
                   ? __hip_atomic_load(rest + i0 + lane * 4 + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT)
                   : 0.0;
      const double scan = wave_scan((x[0] + x[1]) + (x[2] + x[3]));
      each(i0 + lane * 4, x, sum + lane_before(scan));
      sum += lane_value(scan, 63);
    }
    return sum;
  };
  int first = b * kFinish + wave, step = blocks * kFinish;
  double total;
  for (;;) {
    sum_units(first, step);
    // The sums went past the XCD's cache and were waited for, so whoever counts
    // this block among the finished ones finds them; a fence would write that
    // whole cache back, block by block (64 sequences: 71 us in place of 20).
    if (!v.whole) {
      if (threadIdx.x == 0) last_block = atomicAdd(&a.done[s], 1u) == (uint32_t)blocks - 1;
      __syncthreads();
      if (!last_block) return;
    }
    total = running([](int, const double(&)[4], double) {});
    if (total > 0.0 || v.whole) break;
    __syncthreads();  // (every wave has read the sums that the next pass replaces, and all of them the same)
    v.whole = 1;      // nothing left: p itself, by this block
    first = wave;
    step = kFinish;
  }
  if (wave != 0) return;
  // the first unit whose running sum passes the goal; where rounding has left
  // the goal at the whole sum, the last that has any
  const double goal = (double)u * total;
  int unit = -1, last = 0;
  double run = 0.0, last_run = 0.0;
  running([&](int i, const double(&x)[4], double ahead) {
    int hit = -1, any = -1;
    double hit_run = 0.0, any_run = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (x[e] > 0.0) {
        any = i + e;
        any_run = ahead;
        if (hit < 0 && ahead + x[e] > goal) {
          hit = i + e;
          hit_run = ahead;
        }
      }
      ahead += x[e];
    }
    const uint64_t hits = __ballot(hit >= 0), anys = __ballot(any >= 0);
    if (unit < 0 && hits) {
      unit = __builtin_amdgcn_readlane(hit, __builtin_ctzll(hits));
      run = lane_value(hit_run, __builtin_ctzll(hits));
    }
    if (anys) {
      last = __builtin_amdgcn_readlane(any, 63 - __builtin_clzll(anys));
      last_run = lane_value(any_run, 63 - __builtin_clzll(anys));
    }
  });
  if (unit < 0) {
    unit = last;
    run = last_run;
  }
  const int w0 = unit * kUnit + lane * 8;
  double r[8];
  Logits8 x;
  load_residual8<false>(a, v, w0, x);
  residual8(a, v, w0, x, r);
  const double scan = wave_scan(sum8(r));
  const Picked p = pick_wave(pick8(r, run + lane_before(scan), goal, x.at));
  if (lane == 0) write_next(a, s, v, p.hit != kNone ? p.hit : p.last);
}

// ------------------------------------------------------- small vocabularies

// A sequence by one block: V <= kWavePart.
__global__ __launch_bounds__(2 * kSmall * 64) void k_verify_small(VerifyArgs a) {
  constexpr int W = 2 * kSmall;
  __shared__ Verdict shared_v;
  __shared__ double sums[2][W];
  __shared__ Picked picks[W];
  __shared__ uint64_t table[32];
  if (threadIdx.x < 32) table[threadIdx.x] = kPowers[threadIdx.x];
  __syncthreads();
  const int s = blockIdx.x, o0 = a.off[s], o1 = a.off[s + 1], lane = threadIdx.x & 63, wave = wave_index();
  const float u = o1 >= 0 && o1 <= a.n_draft ? a.u[(int64_t)o1 + s] : 0.f;
  judge<kSmall>(a, s, o0, o1, a.draft_logp != nullptr, &shared_v, [&](int j0, int n, RowSum(&rows)[2][kSmall]) {
    const bool prop = wave >= kSmall;
    const int j = j0 + wave % kSmall;
    if (j >= n + (prop ? 0 : 1) || (prop && !a.proposal)) return;
    const void* z = prop ? a.proposal : a.target;
    const int is16 = prop ? a.proposal16 : a.target16;
    const int64_t at = prop ? ((int64_t)o0 + j) * a.ld_p : ((int64_t)o0 + s + j) * a.ld_t;
    const RowSum r = Part<true>(z, is16, at, 0, kWavePart, a.V).sum(table);
    if (lane == 0) rows[prop][wave % kSmall] = r;
  });
  Verdict v = shared_v;
  if (v.bad) {
    if (threadIdx.x == 0) write_bad(a, s, v);
    return;
  }
  const int w0 = (int)threadIdx.x * each_lane(a.V);
  Logits8 x;
  double r[8], total = 0.0, run = 0.0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {  // (a second one where nothing is left: p itself)
    v.whole = pass;
    if (wave == 0 || wave * 512 < a.V) {
      load_residual8<true>(a, v, w0, x);
      residual8(a, v, w0, x, r);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) r[e] = 0.0;
    }
    const double scan = wave_scan(sum8(r));
    if (lane == 63) sums[pass][wave] = scan;
    __syncthreads();
    total = run = 0.0;
    for (int i = 0; i < W; ++i) {
      if (i == wave) run = total;
      total += sums[pass][i];
    }
    run += lane_before(scan);
    if (total > 0.0) break;
  }
  const Picked mine = pick_wave(pick8(r, run, (double)u * total, x.at));
  if (lane == 0) picks[wave] = mine;
  __syncthreads();
  if (threadIdx.x == 0) {
    int hit = kNone, last = -1;
    for (int i = 0; i < W; ++i) {
      hit = min(hit, picks[i].hit);
      last = max(last, picks[i].last);
    }
    write_next(a, s, v, hit != kNone ? hit : last);
  }
}

// Workspace layout (offsets in bytes, 256-aligned).
constexpr int kLeastPart = kWaves * 512;  // a row's parts are no shorter than this
struct VerifyWs {
  size_t rows, rest, done, total;
};
VerifyWs verify_ws(int V, int64_t S, int64_t n_draft) {
  const size_t parts = (size_t)ceil_div(V, kLeastPart), units = (size_t)ceil_div(V, kUnit);
  auto al = [](size_t x) { return (x + 255) / 256 * 256; };
  VerifyWs L{};
  L.rest = L.rows + al((size_t)(S + 2 * n_draft) * parts * sizeof(RowSum));
  L.done = L.rest + al((size_t)S * units * sizeof(double));
  L.total = L.done + al((size_t)S * sizeof(uint32_t));
  return L;
}

}  // namespace

extern "C" {

size_t nmt_verify_workspace_bytes(const nmt_model* m, int32_t S, int32_t n_draft) {
  if (!m || S <= 0 || n_draft < 0) return 0;
  return verify_ws(output_layer(m).V, S, n_draft).total;
}

nmt_status nmt_verify_drafts(nmt_model* m, int32_t S, int32_t n_draft, const int32_t* d_draft_off,
                             const int32_t* d_draft, const void* d_target, int32_t target_type, int64_t ld_target,
                             const void* d_proposal, int32_t proposal_type, int64_t ld_proposal, const float* d_u,
                             int32_t* d_accepted, int32_t* d_next, float* d_draft_logp, float* d_next_logp,
                             void* d_workspace, size_t ws_bytes, void* stream) {
  if (!m) return entry_fail(NMT_EINVAL, "NULL model");
  if (S < 0 || n_draft < 0) return entry_fail(NMT_EINVAL, "negative size");
  if (S == 0) return entry_ok();
  if (!d_draft_off || (n_draft > 0 && !d_draft) || !d_target || !d_u || !d_accepted || !d_next)
    return entry_fail(NMT_EINVAL, "a required device pointer is NULL");
  auto bad_type = [](int32_t t) { return t != NMT_F32 && t != NMT_BF16; };
  if (bad_type(target_type) || (d_proposal && bad_type(proposal_type)))
    return entry_fail(NMT_EINVAL, "unknown element type");
  const OutputLayer layer = output_layer(m);
  const int V = layer.V, cus = layer.cus;
  if (ld_target < V || (d_proposal && ld_proposal < V)) return entry_fail(NMT_EINVAL, "a row stride is below V");
  if (((uintptr_t)d_target & (target_type == NMT_BF16 ? 1 : 3)) ||
      ((uintptr_t)d_proposal & (proposal_type == NMT_BF16 ? 1 : 3)))
    return entry_fail(NMT_EINVAL, "logits must be aligned to their elements");
  // One launch where a wave sums a row by itself and each sequence has a CU
  // (V = 1,000: 8.4 us against 11.1 in two launches for one sequence, 16.4
  // against 15.4 for 512; V = 4,000 and one sequence: 13.8 against 11.5), and
  // for rows too short for the other form's loads.
  const bool small = V < 8 || (V <= kWavePart && S <= cus);
  // Parts as long as the grid still gives each CU four blocks (parts four times
  // as long measured the same), and blocks of a sequence's residual until every
  // wave has one unit or each CU two blocks: each judges its sequence by itself
  // (64 sequences of 50,000 words: 41.4 us a call with three, 37.4 with two, and
  // 39.5 with twice as many blocks of four waves).
  const int64_t n_rows = (int64_t)n_draft + S + (d_proposal ? n_draft : 0);
  int part_len = kWaves * kWavePart;
  while (part_len > kLeastPart && n_rows * ceil_div(V, part_len) < 4 * cus) part_len /= 2;
  const int parts = ceil_div(V, part_len), units = ceil_div(V, kUnit);
  const int64_t n_parts = n_rows * parts;
  const int blocks = (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(units, kFinish), 2 * cus / S));
  // a launch's threads are counted in 32 bits
  if (S >= (1 << 22) || n_parts >= (1 << 24))
    return entry_fail(NMT_EINVAL, "too many rows of logits for one call");
  const VerifyWs L = verify_ws(V, S, n_draft);
  if (!d_workspace || ((uintptr_t)d_workspace & 255)) return entry_fail(NMT_EINVAL, "workspace must be 256-byte aligned");
  if (ws_bytes < L.total) return entry_fail(NMT_EWORKSPACE, "workspace is smaller than nmt_verify_workspace_bytes");
  const nmt_status rc = entry_check_device(m);
  if (rc != NMT_OK) return rc;
  char* ws = (char*)d_workspace;
  const VerifyArgs a{S, n_draft, V, parts, part_len, units, d_draft_off, d_draft, d_target, d_proposal,
                     target_type == NMT_BF16, proposal_type == NMT_BF16, ld_target, ld_proposal, d_u, d_accepted,
                     d_next, d_draft_logp, d_next_logp, (RowSum*)(ws + L.rows), (double*)(ws + L.rest),
                     (uint32_t*)(ws + L.done), error_flag(m)};
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  auto run = [&](auto* kernel, int64_t grid, int threads, auto... args) {
    if (e != hipSuccess) return;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), 0, st, a, args...);
    e = hipGetLastError();
  };
  if (small) {
    run(k_verify_small, S, 2 * kSmall * 64);
  } else {
    run(k_row_sums, n_parts, kWaves * 64);
    run(k_finish, (int64_t)S * blocks, kFinish * 64, blocks);
  }
  if (e != hipSuccess) return entry_hip_fail(e, "nmt_verify_drafts");
  return entry_ok();
}

}  // extern "C"
