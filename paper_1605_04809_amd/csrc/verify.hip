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
#include "draft.hpp"

using namespace nmt;

namespace {

// A row's largest logit and the sum of e^(z - max).
struct RowSum {
  double s;
  float m;
};
__device__ __forceinline__ bool is_distribution(const RowSum& r) {
  return r.m > -INFINITY && r.m < INFINITY && r.s > 0.0 && r.s < INFINITY;
}

struct VerifyArgs {
  int S, n_draft, V;
  const int32_t *off, *draft;
  const void *target, *proposal;  // proposal null: drafts are certain
  int target16, proposal16;
  int64_t ld_t, ld_p;
  const float* u;
  int32_t *accepted, *next;
  float *draft_logp, *next_logp;  // nullable
  RowSum *rows_t, *rows_p;        // workspace
  int* err;
};

__device__ __forceinline__ float logit(const void* z, int is16, int64_t i) {
  return is16 ? (float)((const __bf16*)z)[i] : ((const float*)z)[i];
}

// The sum of v over the block's 256 threads, in a fixed order.
__device__ __forceinline__ double block_sum(double v, double* sh) {
  sh[threadIdx.x] = v;
  __syncthreads();
  for (int n = 128; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) sh[threadIdx.x] += sh[threadIdx.x + n];
    __syncthreads();
  }
  const double r = sh[0];
  __syncthreads();
  return r;
}

// One block per row of target logits, then per row of proposal logits.
__global__ __launch_bounds__(256) void k_row_sums(VerifyArgs a) {
  __shared__ double sh[256];
  __shared__ float mx[256];
  const int n_target = a.n_draft + a.S;
  const bool tgt = (int)blockIdx.x < n_target;
  const int64_t row = tgt ? blockIdx.x : blockIdx.x - n_target;
  const void* z = tgt ? a.target : a.proposal;
  const int is16 = tgt ? a.target16 : a.proposal16;
  const int64_t base = row * (tgt ? a.ld_t : a.ld_p);
  float m = -INFINITY;
  for (int v = threadIdx.x; v < a.V; v += 256) m = fmaxf(m, logit(z, is16, base + v));
  mx[threadIdx.x] = m;
  __syncthreads();
  for (int n = 128; n > 0; n >>= 1) {
    if ((int)threadIdx.x < n) mx[threadIdx.x] = fmaxf(mx[threadIdx.x], mx[threadIdx.x + n]);
    __syncthreads();
  }
  m = mx[0];
  double s = 0.0;
  if (m > -INFINITY)
    for (int v = threadIdx.x; v < a.V; v += 256) s += exp((double)logit(z, is16, base + v) - (double)m);
  s = block_sum(s, sh);
  if (threadIdx.x == 0) (tgt ? a.rows_t : a.rows_p)[row] = RowSum{s, m};
}

// Where a sequence's words come to an end.
struct Verdict {
  int kept, bad;     // bad: no word follows (and which bit of the error flag)
  int64_t t_row, p_row;  // the rows that the next word is drawn from (p_row -1: p itself)
  int32_t cut;       // without proposals: the word that p goes without (-1: none)
};

__device__ __forceinline__ double prob(const void* z, int is16, int64_t i, const RowSum& r) {
  return exp((double)logit(z, is16, i) - (double)r.m) / r.s;
}

__device__ Verdict judge(const VerifyArgs& a, int s) {
  Verdict v{0, 0, 0, -1, -1};
  const int o0 = a.off[s], o1 = a.off[s + 1];
  if (o0 < 0 || o1 < o0 || o1 > a.n_draft) {
    v.bad = 1;
    return v;
  }
  for (int j = 0; j < o1 - o0; ++j) {
    const int64_t tr = (int64_t)o0 + s + j, pr = (int64_t)o0 + j;
    const int32_t d = a.draft[pr];
    const RowSum rt = a.rows_t[tr];
    v.t_row = tr;
    if (d < 0 || d >= a.V) {
      v.bad = 1;
      return v;
    }
    if (!is_distribution(rt)) {
      v.bad = 2;
      return v;
    }
    const double p = prob(a.target, a.target16, tr * a.ld_t + d, rt);
    double q = 1.0;
    if (a.proposal) {
      const RowSum rp = a.rows_p[pr];
      if (!is_distribution(rp)) {
        v.bad = 2;
        return v;
      }
      q = prob(a.proposal, a.proposal16, pr * a.ld_p + d, rp);
    }
    if (!((double)a.u[tr] * q < p)) {
      v.p_row = a.proposal ? pr : -1;
      v.cut = a.proposal ? -1 : d;
      return v;
    }
    ++v.kept;
  }
  v.t_row = (int64_t)o1 + s;
  if (!is_distribution(a.rows_t[v.t_row])) v.bad = 2;
  return v;
}

// One block per sequence: the verdict, then the word after the kept drafts.
__global__ __launch_bounds__(256) void k_verify(VerifyArgs a) {
  __shared__ double sh[256];
  __shared__ Verdict ver;
  __shared__ int word, last;
  const int s = blockIdx.x;
  if (threadIdx.x == 0) {
    ver = judge(a, s);
    word = 0x7fffffff;
    last = -1;
  }
  __syncthreads();
  const Verdict v = ver;
  const int o0 = a.off[s], o1 = a.off[s + 1];
  const bool span_ok = o0 >= 0 && o1 >= o0 && o1 <= a.n_draft;
  if (a.draft_logp && span_ok)
    for (int j = threadIdx.x; j < o1 - o0; j += 256) {
      const int64_t tr = (int64_t)o0 + s + j;
      const int32_t d = a.draft[o0 + j];
      const RowSum r = a.rows_t[tr];
      const bool ok = d >= 0 && d < a.V && is_distribution(r);
      a.draft_logp[o0 + j] =
          ok ? (float)((double)logit(a.target, a.target16, tr * a.ld_t + d) - (double)r.m - log(r.s)) : __builtin_nanf("");
    }
  if (v.bad) {
    if (threadIdx.x == 0) {
      a.accepted[s] = v.kept;
      a.next[s] = -1;
      if (a.next_logp) a.next_logp[s] = __builtin_nanf("");
      atomicOr(a.err, v.bad);
    }
    return;
  }
  const RowSum rt = a.rows_t[v.t_row];
  const RowSum rp = v.p_row >= 0 ? a.rows_p[v.p_row] : RowSum{};
  // a thread's share of the words: a run of consecutive ones
  const int len = (a.V + 255) / 256, v0 = min(a.V, (int)threadIdx.x * len), v1 = min(a.V, v0 + len);
  auto residual = [&](int w, bool whole) {
    double r = prob(a.target, a.target16, v.t_row * a.ld_t + w, rt);
    if (whole) return r;
    if (v.p_row >= 0) r -= prob(a.proposal, a.proposal16, v.p_row * a.ld_p + w, rp);
    return w == v.cut || r < 0.0 ? 0.0 : r;
  };
  bool whole = false;
  double mine = 0.0;
  for (int pass = 0; pass < 2; ++pass) {  // a second one where the residual holds nothing
    mine = 0.0;
    for (int w = v0; w < v1; ++w) mine += residual(w, whole);
    if (whole || block_sum(mine, sh) > 0.0) break;
    whole = true;
  }
  sh[threadIdx.x] = mine;
  __syncthreads();
  double before = 0.0, total = 0.0;
  for (int t = 0; t < 256; ++t) {
    if (t == (int)threadIdx.x) before = total;
    total += sh[t];
  }
  const double goal = (double)a.u[(int64_t)o1 + s] * total;
  double run = before;
  for (int w = v0; w < v1; ++w) {
    const double r = residual(w, whole);
    run += r;
    if (r > 0.0) {
      if (run > goal) {
        atomicMin(&word, w);
        break;
      }
      atomicMax(&last, w);  // (rounding can leave the goal at the whole sum)
    }
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    const int w = word < a.V ? word : last;
    a.accepted[s] = v.kept;
    a.next[s] = w;
    if (a.next_logp)
      a.next_logp[s] = (float)((double)logit(a.target, a.target16, v.t_row * a.ld_t + w) - (double)rt.m - log(rt.s));
  }
}

size_t al256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

extern "C" {

size_t nmt_verify_workspace_bytes(const nmt_model* m, int32_t S, int32_t n_draft) {
  if (!m || S <= 0 || n_draft < 0) return 0;
  return al256(((size_t)n_draft + S) * sizeof(RowSum)) + al256((size_t)n_draft * sizeof(RowSum));
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
  if ((int64_t)S + 2 * (int64_t)n_draft > 0x7fffffff) return entry_fail(NMT_EINVAL, "too many rows of logits");
  const size_t need = nmt_verify_workspace_bytes(m, S, n_draft);
  if (!d_workspace || ((uintptr_t)d_workspace & 255)) return entry_fail(NMT_EINVAL, "workspace must be 256-byte aligned");
  if (ws_bytes < need) return entry_fail(NMT_EWORKSPACE, "workspace is smaller than nmt_verify_workspace_bytes");
  const nmt_status rc = entry_check_device(m);
  if (rc != NMT_OK) return rc;
  char* ws = (char*)d_workspace;
  const VerifyArgs a{S, n_draft, V, d_draft_off, d_draft, d_target, d_proposal, target_type == NMT_BF16,
                     proposal_type == NMT_BF16, ld_target, ld_proposal, d_u, d_accepted, d_next, d_draft_logp,
                     d_next_logp, (RowSum*)ws, (RowSum*)(ws + al256(((size_t)n_draft + S) * sizeof(RowSum))),
                     error_flag(m)};
  hipStream_t st = (hipStream_t)stream;
  hipLaunchKernelGGL(k_row_sums, dim3(n_draft + S + (d_proposal ? n_draft : 0)), dim3(256), 0, st, a);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(k_verify, dim3(S), dim3(256), 0, st, a);
    e = hipGetLastError();
  }
  if (e != hipSuccess) return entry_hip_fail(e, "nmt_verify_drafts");
  return entry_ok();
}

}  // extern "C"
