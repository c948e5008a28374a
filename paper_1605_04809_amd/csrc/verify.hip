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
// running sum.
//
// Large vocabularies take four launches.  k_row_sums reads every row once: a
// wave takes 2,048 logits of one row into registers, all loads in flight at
// once, and leaves their (max, sum) pair.  k_judge merges a sequence's pairs
// and finds where it ends.  k_residual sums what is left of the target over
// 1,024 words a wave, and k_next finds the part, then the word, whose running
// sum passes the random number.  Each stage is spread over the whole chip, so
// one sequence takes no longer than its share of the bandwidth; every sum has
// a fixed order.  Small ones take one launch, a block a sequence (k_verify_small).
#include "draft.hpp"

using namespace nmt;

namespace {

constexpr int kPart = 2048;       // logits of a row that one wave sums
constexpr int kRest = 1024;       // words whose residual one wave sums
constexpr int kWaves = 4;         // waves a block of the streaming kernels
constexpr int kJudge = 8;         // positions a block judges at a time
constexpr int kSmallV = 1024 * 8; // words of the one-launch form: eight a thread

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
  RowSum rt, rp;         // the rows that the next word is drawn from
  int64_t t_row, p_row;  // (p_row -1: the target's alone)
  int32_t kept, bad;     // bad: no word follows (and which bits of the error flag)
  int32_t cut;           // without proposals: the word that p goes without (-1: none)
  int32_t whole;         // the residual holds nothing: p itself
};

struct VerifyArgs {
  int S, n_draft, V, parts, rests;  // parts of a row, and of a residual
  const int32_t *off, *draft;
  const void *target, *proposal;  // proposal null: drafts are certain
  int target16, proposal16;
  int64_t ld_t, ld_p;
  const float* u;
  int32_t *accepted, *next;
  float *draft_logp, *next_logp;  // nullable
  // workspace: parts of the target's rows, then the proposal's; a sequence's
  // verdict; its residual's parts
  RowSum* rows;
  Verdict* verdict;
  double* rest;
  int* err;
};

__device__ __forceinline__ float logit(const void* z, int is16, int64_t i) {
  return is16 ? (float)((const __bf16*)z)[i] : ((const float*)z)[i];
}

// e^x for x <= 0 as 2^n e^r, |r| <= ln 2 / 2, e^r by the polynomial that
// interpolates it at the Chebyshev nodes (off by at most 5.6e-11 of it, and
// exact at 0).  15 64-bit instructions a logit, each at the rate of a 64-bit
// multiply-add: 2 T logits/s, which keeps up with 8 TB/s of fp32 ones.  The
// odds that a sum's error moves a decision are its part of the distance
// between two borders: at most 5.6e-11 for a draft, and 1e-5 even for a word
// out of 100,000 equal ones if every error had the same sign.
__device__ __forceinline__ double exp_neg(double x) {
  constexpr double kShift = 6755399441055744.0;  // 1.5 * 2^52: n comes out in the sum's low bits
  const double d = fmax(x, -760.0);
  const double t = fma(d, 1.4426950408889634, kShift);
  const double r = fma(t - kShift, -0.6931471805599453, d);
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

// maximum() returns NaN if either is (fmaxf does not).
__device__ __forceinline__ float maximum(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float wave_maximum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v = maximum(v, __shfl_xor(v, o, 64));
  return v;
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Inclusive running sums over the wave's lanes.
__device__ __forceinline__ double wave_scan(double v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const double u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

// Eight consecutive logits at z[i], those from n on as -infinity; any
// alignment of the elements' own.  (The type is a branch here, the same for
// the whole wave, and not a form of each kernel: their code would double, and
// a block that runs once waits for its instructions as for its data.)
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
__device__ __forceinline__ void load8(const void* z, int is16, int64_t i, int n, float (&x)[8]) {
  if (n < 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < n ? logit(z, is16, i + e) : -INFINITY;
  } else if (is16) {
    const bf16x8u a = *(const bf16x8u*)((const __bf16*)z + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)a[e];
  } else {
    const f32x4u a = *(const f32x4u*)((const float*)z + i), b = *(const f32x4u*)((const float*)z + i + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < 4 ? a[e] : b[e - 4];
  }
}

// ------------------------------------------------------------- row sums

// The pair of one part of a row, by one wave: the n <= kPart logits at z.
constexpr int kSteps = kPart / 512;  // eight logits a lane and step
__device__ __forceinline__ RowSum part_sum(const void* z, int is16, int64_t at, int n) {
  const int lane = threadIdx.x & 63;
  float x[kSteps][8];
  auto load = [&](int type) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) load8(z, type, at + i * 512 + lane * 8, n - (i * 512 + lane * 8), x[i]);
  };
  if (is16)
    load(1);
  else
    load(0);
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kSteps; ++i)
#pragma unroll
    for (int e = 0; e < 8; ++e) m = maximum(m, x[i][e]);
  m = wave_maximum(m);
  double s = 0.0;
  if (m > -INFINITY && m < INFINITY) {
    double s1 = 0.0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i * 512 >= n) break;  // (a short row has few steps)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        s += exp_neg((double)x[i][e] - (double)m);
        s1 += exp_neg((double)x[i][e + 1] - (double)m);
      }
    }
    s = wave_sum(s + s1);
  }
  return RowSum{s, m};
}

__device__ __forceinline__ RowSum merge(const RowSum& a, const RowSum& b) {
  const float m = maximum(a.m, b.m);
  if (!(m > -INFINITY && m < INFINITY)) return RowSum{0.0, m};
  return RowSum{a.s * exp_neg((double)a.m - (double)m) + b.s * exp_neg((double)b.m - (double)m), m};
}

// A row's pair from its parts', by one wave.
__device__ __forceinline__ RowSum merge_parts(const RowSum* r, int parts) {
  const int lane = threadIdx.x & 63;
  RowSum mine = lane < parts ? r[lane] : RowSum{0.0, -INFINITY};
  for (int i = lane + 64; i < parts; i += 64) mine = merge(mine, r[i]);
  const float m = wave_maximum(mine.m);
  const bool ok = m > -INFINITY && m < INFINITY;
  return RowSum{wave_sum(ok ? mine.s * exp_neg((double)mine.m - (double)m) : 0.0), m};
}

// One wave per part of a row.
__global__ __launch_bounds__(kWaves * 64) void k_row_sums(VerifyArgs a, int64_t n_all) {
  const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (id >= n_all) return;
  const int64_t row = id / a.parts;
  const int part = (int)(id % a.parts), n = min(kPart, a.V - part * kPart);
  const int64_t n_target = (int64_t)a.n_draft + a.S;
  const bool tgt = row < n_target;
  const int64_t at = (tgt ? row * a.ld_t : (row - n_target) * a.ld_p) + (int64_t)part * kPart;
  const RowSum r = part_sum(tgt ? a.target : a.proposal, tgt ? a.target16 : a.proposal16, at, n);
  if ((threadIdx.x & 63) == 0) a.rows[id] = r;
}

// --------------------------------------------------------------- verdict

// The verdict on sequence s, by a block of 2 kJudge waves: kJudge positions at
// a time, a wave for each's target row and one for its proposal row
// (row_sum(is_target, row)), then the first wave with a lane a position.  Log p
// of each draft goes out too, and every position is looked at for it.  The
// block's verdict is in *out after the call.
template <class RowSumOf>
__device__ __forceinline__ void judge(const VerifyArgs& a, int s, int o0, int o1, Verdict* out, RowSumOf&& row_sum) {
  __shared__ RowSum rows[2][kJudge];
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
  for (int j0 = 0; j0 <= n; j0 += kJudge) {
    const bool prop = wave >= kJudge;
    const int jw = j0 + wave % kJudge;
    if (jw < n + (prop ? 0 : 1) && (!prop || a.proposal)) {
      const RowSum r = row_sum(!prop, prop ? (int64_t)o0 + jw : (int64_t)o0 + s + jw);
      if (lane == 0) rows[prop][wave % kJudge] = r;
    }
    // what else a position is judged by, on its way meanwhile
    const int j = j0 + lane;
    const bool pos = wave == 0 && lane < kJudge && j <= n, has_p = pos && j < n && a.proposal;
    const int64_t tr = (int64_t)o0 + s + j, pr = (int64_t)o0 + j;
    const int32_t d = pos && j < n ? a.draft[pr] : 0;
    const float u = pos ? a.u[tr] : 0.f;
    const bool d_ok = d >= 0 && d < a.V;
    const float zt = pos ? logit(a.target, a.target16, tr * a.ld_t + (d_ok ? d : 0)) : 0.f;
    const float zp = has_p ? logit(a.proposal, a.proposal16, pr * a.ld_p + (d_ok ? d : 0)) : 0.f;
    __syncthreads();
    if (wave == 0) {
      const RowSum rt = rows[0][lane % kJudge], rp = has_p ? rows[1][lane % kJudge] : RowSum{1.0, 0.f};
      const bool t_ok = is_distribution(rt);
      const int bad = !d_ok ? 1 : !t_ok || !is_distribution(rp) ? 2 : 0;
      const double p = exp_neg((double)zt - (double)rt.m) / rt.s;
      const double q = has_p ? exp_neg((double)zp - (double)rp.m) / rp.s : 1.0;
      const bool end = pos && (j == n || bad || !((double)u * q < p));
      const uint64_t ends = __ballot(end);
      if (!done && ends && lane == __builtin_ctzll(ends)) {
        *out = Verdict{rt, rp, tr, has_p ? pr : -1, j, bad, j < n && !a.proposal ? d : -1, 0};
        done = 1;
      }
      if (pos && j < n && a.draft_logp)
        a.draft_logp[pr] = d_ok && t_ok ? (float)((double)zt - (double)rt.m - log(rt.s)) : __builtin_nanf("");
    }
    __syncthreads();
    if (done && !a.draft_logp) break;
  }
}

// One block a sequence.
__global__ __launch_bounds__(2 * kJudge * 64) void k_judge(VerifyArgs a) {
  const int s = blockIdx.x;
  const int64_t n_target = (int64_t)a.n_draft + a.S;
  judge(a, s, a.off[s], a.off[s + 1], a.verdict + s, [&](bool tgt, int64_t row) {
    return merge_parts(a.rows + (tgt ? row : n_target + row) * a.parts, a.parts);
  });
}

// A sequence that no word follows.
__device__ __forceinline__ void write_bad(const VerifyArgs& a, int s, const Verdict& v) {
  a.accepted[s] = v.kept;
  a.next[s] = -1;
  if (a.next_logp) a.next_logp[s] = __builtin_nanf("");
  atomicOr(a.err, v.bad);
}

// -------------------------------------------------------------- residual

// What is left of words w0 .. w0 + 7 for the draw (nothing of those past V).
__device__ __forceinline__ void residual8(const VerifyArgs& a, const Verdict& v, int w0, double (&r)[8]) {
  float xt[8], xp[8];
  const bool minus = v.p_row >= 0 && !v.whole;
  load8(a.target, a.target16, v.t_row * a.ld_t + w0, a.V - w0, xt);
  if (minus) load8(a.proposal, a.proposal16, v.p_row * a.ld_p + w0, a.V - w0, xp);
  const double it = 1.0 / v.rt.s;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = exp_neg((double)xt[e] - (double)v.rt.m) * it;
  if (minus) {
    const double ip = 1.0 / v.rp.s;
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = fmax(r[e] - exp_neg((double)xp[e] - (double)v.rp.m) * ip, 0.0);
  } else if (v.cut >= 0 && !v.whole) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r[e] = w0 + e == v.cut ? 0.0 : r[e];
  }
}
__device__ __forceinline__ double sum8(const double (&r)[8]) {
  return ((r[0] + r[1]) + (r[2] + r[3])) + ((r[4] + r[5]) + (r[6] + r[7]));
}

// The residual's sum over part p of the words, by one wave.
__device__ __forceinline__ double rest_sum(const VerifyArgs& a, const Verdict& v, int part) {
  double sum = 0.0;
#pragma unroll 1
  for (int i = 0; i < kRest / 512; ++i) {
    double r[8];
    residual8(a, v, part * kRest + i * 512 + (threadIdx.x & 63) * 8, r);
    sum += sum8(r);
  }
  return wave_sum(sum);
}

// One wave per part of a sequence's words.
__global__ __launch_bounds__(kWaves * 64) void k_residual(VerifyArgs a, int64_t n_all) {
  const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  if (id >= n_all) return;
  const int s = (int)(id / a.rests);
  const Verdict v = a.verdict[s];
  if (v.bad) return;
  const double sum = rest_sum(a, v, (int)(id % a.rests));
  if ((threadIdx.x & 63) == 0) a.rest[id] = sum;
}

// The first word of the block's (eight a thread from w0, whose residuals are
// r and whose running sum starts at `run`) whose running sum passes the goal;
// where rounding has left the goal at the whole sum, the last that has any.
template <int NW>
__device__ __forceinline__ int pick(const double (&r)[8], double run, double goal, int w0) {
  __shared__ int word[NW], last[NW];
  int hit_w = 0x7fffffff, last_w = -1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    run += r[e];
    if (r[e] > 0.0) {
      if (run > goal && hit_w == 0x7fffffff) hit_w = w0 + e;
      last_w = w0 + e;
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    hit_w = min(hit_w, __shfl_xor(hit_w, o, 64));
    last_w = max(last_w, __shfl_xor(last_w, o, 64));
  }
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    word[wave] = hit_w;
    last[wave] = last_w;
  }
  __syncthreads();
  for (int i = 0; i < NW; ++i) {
    hit_w = min(hit_w, word[i]);
    last_w = max(last_w, last[i]);
  }
  return hit_w == 0x7fffffff ? last_w : hit_w;
}

// The sum of the block's values before this thread's, and all of them.
template <int NW>
__device__ __forceinline__ double block_before(double mine, double* total) {
  __shared__ double sums[NW];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const double sc = wave_scan(mine), up = __shfl_up(sc, 1, 64);
  __syncthreads();
  if (lane == 63) sums[wave] = sc;
  __syncthreads();
  double before = 0.0, sum = 0.0;
  for (int i = 0; i < NW; ++i) {
    if (i == wave) before = sum;
    sum += sums[i];
  }
  *total = sum;
  return before + (lane > 0 ? up : 0.0);
}

__device__ __forceinline__ void write_next(const VerifyArgs& a, int s, const Verdict& v, int w) {
  a.accepted[s] = v.kept;
  a.next[s] = w;
  if (a.next_logp)
    a.next_logp[s] = (float)((double)logit(a.target, a.target16, v.t_row * a.ld_t + w) - (double)v.rt.m - log(v.rt.s));
}

// The sequence's word from its residual's parts.  One block a sequence, eight
// words of the part a thread.
constexpr int kNextWaves = kRest / 512;
__global__ __launch_bounds__(kNextWaves * 64) void k_next(VerifyArgs a) {
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Verdict v = a.verdict[s];
  if (v.bad) {
    if (threadIdx.x == 0) write_bad(a, s, v);
    return;
  }
  double* rest = a.rest + (int64_t)s * a.rests;
  const double u = a.u[(int64_t)a.off[s + 1] + s];
  auto running = [&](auto&& each) {  // each(part, its sum, the sum before it); returns the whole sum
    double sum = 0.0;
    for (int i = 0; i < a.rests; i += 64) {
      const double x = i + lane < a.rests ? rest[i + lane] : 0.0;
      const double sc = wave_scan(x);
      const double up = __shfl_up(sc, 1, 64);
      each(i, x, sum + (lane > 0 ? up : 0.0));
      sum += __shfl(sc, 63, 64);
    }
    return sum;
  };
  double total = running([](int, double, double) {});
  if (!(total > 0.0)) {  // nothing left: p itself
    v.whole = 1;
    for (int p = wave; p < a.rests; p += kNextWaves) {
      const double sum = rest_sum(a, v, p);
      if (lane == 0) rest[p] = sum;
    }
    __syncthreads();
    total = running([](int, double, double) {});
  }
  const double goal = u * total;
  int part = -1, last_part = 0;
  double before = 0.0, last_before = 0.0;
  running([&](int i, double x, double ahead) {
    const uint64_t hit = __ballot(x > 0.0 && ahead + x > goal), any = __ballot(x > 0.0);
    if (part < 0 && hit) {
      const int l = __builtin_ctzll(hit);
      part = i + l;
      before = __shfl(ahead, l, 64);
    }
    if (any) {
      const int l = 63 - __builtin_clzll(any);
      last_part = i + l;
      last_before = __shfl(ahead, l, 64);
    }
  });
  if (part < 0) {  // (rounding can leave the goal at the whole sum)
    part = last_part;
    before = last_before;
  }
  const int w0 = part * kRest + (int)threadIdx.x * 8;
  double r[8], all;
  residual8(a, v, w0, r);
  const double ahead = block_before<kNextWaves>(sum8(r), &all);
  const int w = pick<kNextWaves>(r, before + ahead, goal, w0);
  if (threadIdx.x == 0) write_next(a, s, v, w);
}

// ------------------------------------------------------- small vocabularies

// A sequence by one block: V <= kSmallV.
__global__ __launch_bounds__(2 * kJudge * 64) void k_verify_small(VerifyArgs a) {
  __shared__ Verdict shared_v;
  const int s = blockIdx.x, o0 = a.off[s], o1 = a.off[s + 1];
  judge(a, s, o0, o1, &shared_v, [&](bool tgt, int64_t row) {
    const void* z = tgt ? a.target : a.proposal;
    const int is16 = tgt ? a.target16 : a.proposal16;
    const int64_t at = row * (tgt ? a.ld_t : a.ld_p);
    RowSum r{0.0, -INFINITY};
#pragma unroll 1
    for (int i = 0; i < a.V; i += kPart) {
      const RowSum p = part_sum(z, is16, at + i, min(kPart, a.V - i));
      r = i ? merge(r, p) : p;
    }
    return r;
  });
  Verdict v = shared_v;
  if (v.bad) {
    if (threadIdx.x == 0) write_bad(a, s, v);
    return;
  }
  const int w0 = (int)threadIdx.x * 8;
  double r[8], total, ahead;
  residual8(a, v, w0, r);
  ahead = block_before<2 * kJudge>(sum8(r), &total);
  if (!(total > 0.0)) {  // nothing left: p itself
    v.whole = 1;
    residual8(a, v, w0, r);
    ahead = block_before<2 * kJudge>(sum8(r), &total);
  }
  const int w = pick<2 * kJudge>(r, ahead, (double)a.u[(int64_t)o1 + s] * total, w0);
  if (threadIdx.x == 0) write_next(a, s, v, w);
}

// Workspace layout (offsets in bytes, 256-aligned).
struct VerifyWs {
  size_t rows, verdict, rest, total;
};
VerifyWs verify_ws(int V, int64_t S, int64_t n_draft) {
  const size_t parts = (size_t)ceil_div(V, kPart), rests = (size_t)ceil_div(V, kRest);
  auto al = [](size_t x) { return (x + 255) / 256 * 256; };
  VerifyWs L{};
  L.verdict = L.rows + al((size_t)(S + 2 * n_draft) * parts * sizeof(RowSum));
  L.rest = L.verdict + al((size_t)S * sizeof(Verdict));
  L.total = L.rest + al((size_t)S * rests * sizeof(double));
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
  const int V = output_layer(m).V;
  if (ld_target < V || (d_proposal && ld_proposal < V)) return entry_fail(NMT_EINVAL, "a row stride is below V");
  if (((uintptr_t)d_target & (target_type == NMT_BF16 ? 1 : 3)) ||
      ((uintptr_t)d_proposal & (proposal_type == NMT_BF16 ? 1 : 3)))
    return entry_fail(NMT_EINVAL, "logits must be aligned to their elements");
  const int parts = ceil_div(V, kPart), rests = ceil_div(V, kRest);
  const int64_t n_rows = (int64_t)n_draft + S + (d_proposal ? n_draft : 0), n_parts = n_rows * parts;
  const int64_t n_rests = (int64_t)S * rests;
  auto blocks = [](int64_t waves) { return (waves + kWaves - 1) / kWaves; };
  if (blocks(n_parts) > 0x7fffffff || blocks(n_rests) > 0x7fffffff)
    return entry_fail(NMT_EINVAL, "too many rows of logits for one call");
  const VerifyWs L = verify_ws(V, S, n_draft);
  if (!d_workspace || ((uintptr_t)d_workspace & 255)) return entry_fail(NMT_EINVAL, "workspace must be 256-byte aligned");
  if (ws_bytes < L.total) return entry_fail(NMT_EWORKSPACE, "workspace is smaller than nmt_verify_workspace_bytes");
  const nmt_status rc = entry_check_device(m);
  if (rc != NMT_OK) return rc;
  char* ws = (char*)d_workspace;
  const VerifyArgs a{S, n_draft, V, parts, rests, d_draft_off, d_draft, d_target, d_proposal, target_type == NMT_BF16,
                     proposal_type == NMT_BF16, ld_target, ld_proposal, d_u, d_accepted, d_next, d_draft_logp,
                     d_next_logp, (RowSum*)(ws + L.rows), (Verdict*)(ws + L.verdict), (double*)(ws + L.rest),
                     error_flag(m)};
  hipStream_t st = (hipStream_t)stream;
  hipError_t e = hipSuccess;
  auto run = [&](auto* kernel, int64_t grid, int threads, auto... args) {
    if (e != hipSuccess) return;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(threads), 0, st, a, args...);
    e = hipGetLastError();
  };
  if (V <= kSmallV) {
    run(k_verify_small, S, 2 * kJudge * 64);
  } else {
    run(k_row_sums, blocks(n_parts), kWaves * 64, n_parts);
    run(k_judge, S, 2 * kJudge * 64);
    run(k_residual, blocks(n_rests), kWaves * 64, n_rests);
    run(k_next, S, kNextWaves * 64);
  }
  if (e != hipSuccess) return entry_hip_fail(e, "nmt_verify_drafts");
  return entry_ok();
}

}  // extern "C"
