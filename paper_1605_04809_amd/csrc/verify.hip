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
// Three launches.  k_row_sums reads every row once: a wave takes 2,048 logits
// of one row into registers, all loads in flight at once, and leaves their
// (max, sum) pair.  k_residual judges its sequence from those pairs (each
// block by itself, all positions at once) and sums the residual over its own
// words, and k_next finds the word from the parts' sums.  A sequence's parts
// are spread over the chip, so that one sequence over a large vocabulary takes
// no longer than its share of the bandwidth; every sum has a fixed order.
#include <type_traits>

#include "draft.hpp"

using namespace nmt;

namespace {

constexpr int kPart = 2048;       // logits of a row that one wave sums
constexpr int kWaves = 4;         // waves a block

// A row's (or a part's) largest logit and the sum of e^(z - max).  A NaN makes
// both NaN, and a row of nothing but -infinity has max -infinity and sum 0.
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
  int32_t whole;         // the residual holds nothing: p itself (set by k_next)
};

struct VerifyArgs {
  int S, n_draft, V, parts;       // parts of a row
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

// e^x for x <= 0 (or NaN's stand-in): 2^(x log2 e) as 2^n times the power
// series of 2^f, |f| <= 1/2, whose eleventh-order remainder is 2.2e-13 of it.
// 18 64-bit instructions a logit, at which the chip keeps up with its memory
// (8 TB/s of fp32 logits).
__device__ __forceinline__ double exp_neg(double x) {
  const double t = fmax(x * 1.4426950408889634, -1100.0);
  const double n = rint(t);
  const double r = (t - n) * 0.6931471805599453;
  double p = 1.0 / 3628800.0;
  p = fma(p, r, 1.0 / 362880.0);
  p = fma(p, r, 1.0 / 40320.0);
  p = fma(p, r, 1.0 / 5040.0);
  p = fma(p, r, 1.0 / 720.0);
  p = fma(p, r, 1.0 / 120.0);
  p = fma(p, r, 1.0 / 24.0);
  p = fma(p, r, 1.0 / 6.0);
  p = fma(p, r, 0.5);
  p = fma(p, r, 1.0);
  p = fma(p, r, 1.0);
  return ldexp(p, (int)n);
}

__device__ __forceinline__ double prob(float z, const RowSum& r) {
  return exp_neg((double)z - (double)r.m) / r.s;
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

// Eight consecutive logits at z[i], those from n on as -infinity; any
// alignment of the elements' own.
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
__device__ __forceinline__ void load8(const float* z, int64_t i, int n, float (&x)[8]) {
  if (n >= 8) {
    const f32x4u a = *(const f32x4u*)(z + i), b = *(const f32x4u*)(z + i + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < 4 ? a[e] : b[e - 4];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < n ? z[i + e] : -INFINITY;
  }
}
__device__ __forceinline__ void load8(const __bf16* z, int64_t i, int n, float (&x)[8]) {
  if (n >= 8) {
    const bf16x8u a = *(const bf16x8u*)(z + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)a[e];
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = e < n ? (float)z[i + e] : -INFINITY;
  }
}

// The pair of one part of a row, by one wave: the n <= kPart logits at z.
constexpr int kSteps = kPart / 512;  // eight logits a lane and step
template <class T>
__device__ __forceinline__ RowSum part_sum(const T* z, int n) {
  const int lane = threadIdx.x & 63;
  float x[kSteps][8];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) load8(z, i * 512 + lane * 8, n - (i * 512 + lane * 8), x[i]);
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
    for (int i = 0; i < kSteps; ++i)
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        s += exp_neg((double)x[i][e] - (double)m);
        s1 += exp_neg((double)x[i][e + 1] - (double)m);
      }
    s = wave_sum(s + s1);
  }
  return RowSum{s, m};
}

// A row's pair from its parts', by one wave.
__device__ __forceinline__ RowSum merge_parts(const RowSum* r, int parts) {
  const int lane = threadIdx.x & 63;
  RowSum mine{0.0, -INFINITY};
  for (int i = lane; i < parts; i += 64) {
    const RowSum o = r[i];
    const float m = maximum(mine.m, o.m);
    if (m > -INFINITY && m < INFINITY)
      mine.s = mine.s * exp_neg((double)mine.m - (double)m) + o.s * exp_neg((double)o.m - (double)m);
    mine.m = m;
  }
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
  const void* z = tgt ? a.target : a.proposal;
  const RowSum r = (tgt ? a.target16 : a.proposal16) ? part_sum((const __bf16*)z + at, n)
                                                     : part_sum((const float*)z + at, n);
  if ((threadIdx.x & 63) == 0) a.rows[id] = r;
}

// The verdict on sequence s by a block of kWaves waves, kWaves positions at a
// time.  With write, log p of each draft goes out too (and every position is
// looked at for it).
__device__ Verdict judge(const VerifyArgs& a, int s, bool write) {
  __shared__ Verdict sh[kWaves];
  __shared__ int stop[kWaves];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int o0 = a.off[s], o1 = a.off[s + 1];
  Verdict v{};
  if (o0 < 0 || o1 < o0 || o1 > a.n_draft) {
    v.bad = 1;
    return v;
  }
  const int64_t n_target = (int64_t)a.n_draft + a.S;
  const int n = o1 - o0;
  bool found = false;
  for (int j0 = 0; j0 <= n && !(found && !write); j0 += kWaves) {
    const int j = j0 + wave;
    if (j <= n) {
      const int64_t tr = (int64_t)o0 + s + j, pr = (int64_t)o0 + j;
      Verdict w{};
      w.kept = j;
      w.t_row = tr;
      w.p_row = -1;
      w.cut = -1;
      const bool has_p = j < n && a.proposal;
      const int32_t d = j < n ? a.draft[pr] : 0;
      const bool d_ok = d >= 0 && d < a.V;
      const float zt = logit(a.target, a.target16, tr * a.ld_t + (d_ok ? d : 0));
      const float zp = has_p ? logit(a.proposal, a.proposal16, pr * a.ld_p + (d_ok ? d : 0)) : 0.f;
      w.rt = merge_parts(a.rows + tr * a.parts, a.parts);
      if (has_p) w.rp = merge_parts(a.rows + (n_target + pr) * a.parts, a.parts);
      const bool t_ok = is_distribution(w.rt);
      if (!d_ok)
        w.bad = 1;
      else if (!t_ok || (has_p && !is_distribution(w.rp)))
        w.bad = 2;
      bool end = true;
      if (j < n) {
        if (!w.bad) {
          const double q = has_p ? prob(zp, w.rp) : 1.0;
          end = !((double)a.u[tr] * q < prob(zt, w.rt));  // (a NaN ends it too)
          w.p_row = has_p ? pr : -1;
          w.cut = has_p ? -1 : d;
        }
        if (write && lane == 0)
          a.draft_logp[pr] = d_ok && t_ok ? (float)((double)zt - (double)w.rt.m - log(w.rt.s)) : __builtin_nanf("");
      }
      if (lane == 0) {
        sh[wave] = w;
        stop[wave] = end;
      }
    } else if (lane == 0) {
      stop[wave] = 0;
    }
    __syncthreads();
    for (int w = 0; w < kWaves && !found; ++w)
      if (stop[w]) {
        v = sh[w];
        found = true;
      }
    __syncthreads();
  }
  return v;
}

// What is left of word w for the draw (it, ip: the rows' sums' reciprocals).
__device__ __forceinline__ double residual(const Verdict& v, double it, double ip, float zt, float zp, int w) {
  double r = exp_neg((double)zt - (double)v.rt.m) * it;
  if (v.whole) return r;
  if (v.p_row >= 0) r -= exp_neg((double)zp - (double)v.rp.m) * ip;
  return w == v.cut || r < 0.0 ? 0.0 : r;
}
template <class TT, class TP>
__device__ __forceinline__ void residual8(const VerifyArgs& a, const Verdict& v, int w0, int n, double (&r)[8]) {
  float xt[8], xp[8];
  load8((const TT*)a.target, v.t_row * a.ld_t + w0, n, xt);
  if (v.p_row >= 0) {
    load8((const TP*)a.proposal, v.p_row * a.ld_p + w0, n, xp);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) xp[e] = 0.f;
  }
  const double it = 1.0 / v.rt.s, ip = v.p_row >= 0 ? 1.0 / v.rp.s : 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = residual(v, it, ip, xt[e], xp[e], w0 + e);
}
// f with the two matrices' element types.
template <class F>
__device__ __forceinline__ void with_types(const VerifyArgs& a, F&& f) {
  if (a.target16) {
    if (a.proposal16)
      f((__bf16*)nullptr, (__bf16*)nullptr);
    else
      f((__bf16*)nullptr, (float*)nullptr);
  } else {
    if (a.proposal16)
      f((float*)nullptr, (__bf16*)nullptr);
    else
      f((float*)nullptr, (float*)nullptr);
  }
}

// The sum of the residual over part p of sequence s's words, by one wave.
__device__ __forceinline__ double rest_sum(const VerifyArgs& a, const Verdict& v, int part) {
  const int lane = threadIdx.x & 63;
  double sum = 0.0;
  with_types(a, [&](auto* tt, auto* tp) {
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int w0 = part * kPart + i * 512 + lane * 8;
      double r[8];
      residual8<std::remove_pointer_t<decltype(tt)>, std::remove_pointer_t<decltype(tp)>>(a, v, w0, a.V - w0, r);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum += r[e];
    }
  });
  return wave_sum(sum);
}

// One wave per part of a sequence's words, kWaves parts a block: the verdict
// (written by the sequence's first block), then the residual's sums.
__global__ __launch_bounds__(kWaves * 64) void k_residual(VerifyArgs a, int blocks) {
  const int s = blockIdx.x / blocks, b = blockIdx.x % blocks;
  const Verdict v = judge(a, s, b == 0 && a.draft_logp);
  if (b == 0 && threadIdx.x == 0) a.verdict[s] = v;
  const int part = b * kWaves + (threadIdx.x >> 6);
  if (v.bad || part >= a.parts) return;
  const double sum = rest_sum(a, v, part);
  if ((threadIdx.x & 63) == 0) a.rest[(int64_t)s * a.parts + part] = sum;
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

// The sequence's word: the part whose running sum passes the goal, then the
// word within it.  One block a sequence, a wave per 512 words of the part.
__global__ __launch_bounds__(kSteps * 64) void k_next(VerifyArgs a) {
  __shared__ double step_sum[kSteps];
  __shared__ int word[kSteps], last[kSteps];
  const int s = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Verdict v = a.verdict[s];
  if (v.bad) {
    if (threadIdx.x == 0) {
      a.accepted[s] = v.kept;
      a.next[s] = -1;
      if (a.next_logp) a.next_logp[s] = __builtin_nanf("");
      atomicOr(a.err, v.bad);
    }
    return;
  }
  double* rest = a.rest + (int64_t)s * a.parts;
  auto running = [&](auto&& each) {  // each(part, its sum, the sum before it); returns the whole sum
    double sum = 0.0;
    for (int i = 0; i < a.parts; i += 64) {
      const double x = i + lane < a.parts ? rest[i + lane] : 0.0;
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
    for (int p = wave; p < a.parts; p += kSteps) {
      const double sum = rest_sum(a, v, p);
      if (lane == 0) rest[p] = sum;
    }
    __syncthreads();
    total = running([](int, double, double) {});
  }
  const double goal = (double)a.u[(int64_t)a.off[s + 1] + s] * total;
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
  const int w0 = part * kPart + wave * 512 + lane * 8;
  double r[8], mine = 0.0;
  with_types(a, [&](auto* tt, auto* tp) {
    residual8<std::remove_pointer_t<decltype(tt)>, std::remove_pointer_t<decltype(tp)>>(a, v, w0, a.V - w0, r);
  });
#pragma unroll
  for (int e = 0; e < 8; ++e) mine += r[e];
  const double sc = wave_scan(mine), up = __shfl_up(sc, 1, 64);
  if (lane == 63) step_sum[wave] = sc;
  __syncthreads();
  double run = before;
  for (int w = 0; w < wave; ++w) run += step_sum[w];
  run += lane > 0 ? up : 0.0;
  int hit_w = a.V, last_w = -1;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    run += r[e];
    if (r[e] > 0.0) {
      if (run > goal && hit_w == a.V) hit_w = w0 + e;
      last_w = w0 + e;
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    hit_w = min(hit_w, __shfl_xor(hit_w, o, 64));
    last_w = max(last_w, __shfl_xor(last_w, o, 64));
  }
  if (lane == 0) {
    word[wave] = hit_w;
    last[wave] = last_w;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    int w = a.V, l = -1;
    for (int i = 0; i < kSteps; ++i) {
      w = min(w, word[i]);
      l = max(l, last[i]);
    }
    if (w == a.V) w = l;
    a.accepted[s] = v.kept;
    a.next[s] = w;
    if (a.next_logp)
      a.next_logp[s] = (float)((double)logit(a.target, a.target16, v.t_row * a.ld_t + w) - (double)v.rt.m - log(v.rt.s));
  }
}

// Workspace layout (offsets in bytes, 256-aligned).
struct VerifyWs {
  size_t rows, verdict, rest, total;
};
VerifyWs verify_ws(int V, int64_t S, int64_t n_draft) {
  const size_t parts = (size_t)ceil_div(V, kPart);
  auto al = [](size_t x) { return (x + 255) / 256 * 256; };
  VerifyWs L{};
  L.verdict = L.rows + al((size_t)(S + 2 * n_draft) * parts * sizeof(RowSum));
  L.rest = L.verdict + al((size_t)S * sizeof(Verdict));
  L.total = L.rest + al((size_t)S * parts * sizeof(double));
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
  const int parts = ceil_div(V, kPart), res_blocks = ceil_div(parts, kWaves);
  const int64_t n_rows = (int64_t)n_draft + S + (d_proposal ? n_draft : 0), n_parts = n_rows * parts;
  if ((n_parts + kWaves - 1) / kWaves > 0x7fffffff || (int64_t)S * res_blocks > 0x7fffffff)
    return entry_fail(NMT_EINVAL, "too many rows of logits for one call");
  const VerifyWs L = verify_ws(V, S, n_draft);
  if (!d_workspace || ((uintptr_t)d_workspace & 255)) return entry_fail(NMT_EINVAL, "workspace must be 256-byte aligned");
  if (ws_bytes < L.total) return entry_fail(NMT_EWORKSPACE, "workspace is smaller than nmt_verify_workspace_bytes");
  const nmt_status rc = entry_check_device(m);
  if (rc != NMT_OK) return rc;
  char* ws = (char*)d_workspace;
  const VerifyArgs a{S, n_draft, V, parts, d_draft_off, d_draft, d_target, d_proposal, target_type == NMT_BF16,
                     proposal_type == NMT_BF16, ld_target, ld_proposal, d_u, d_accepted, d_next, d_draft_logp,
                     d_next_logp, (RowSum*)(ws + L.rows), (Verdict*)(ws + L.verdict), (double*)(ws + L.rest),
                     error_flag(m)};
  hipStream_t st = (hipStream_t)stream;
  hipLaunchKernelGGL(k_row_sums, dim3((unsigned)((n_parts + kWaves - 1) / kWaves)), dim3(kWaves * 64), 0, st, a, n_parts);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(k_residual, dim3((unsigned)(S * res_blocks)), dim3(kWaves * 64), 0, st, a, res_blocks);
    e = hipGetLastError();
  }
  if (e == hipSuccess) {
    hipLaunchKernelGGL(k_next, dim3(S), dim3(kSteps * 64), 0, st, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return entry_hip_fail(e, "nmt_verify_drafts");
  return entry_ok();
}

}  // extern "C"
