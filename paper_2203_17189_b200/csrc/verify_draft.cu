// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Sequence s has n drafted tokens x_0 .. x_{n-1}, drawn from draft_0 .. draft_{n-1} (or, without draft probabilities,
// given with certainty: draft_i is one at x_i and zero elsewhere).  x_i is accepted while u_i draft_i(x_i) < target_i(x_i),
// i.e. with probability min(1, target / draft).  Behind the a accepted tokens one more is drawn: from
// max(target_a - draft_a, 0) when x_a was refused, from target_n when none was.  The tokens then follow the target's
// distribution.  The draw inverts the cumulative sum: the first v with sum_{i <= v} r_i > u sum_i r_i.
//
// All arithmetic on the probabilities is float64 (a product of two float32 values and a difference are exact there, a sum
// of 10^5 of them is off by 10^-16 of the total), so the outcome does not depend on the order of the sums.
//
// Bound: latency.  Only the row behind the last accepted token is read, once: 2 V values per sequence.  A cluster of CTAs
// takes one sequence; every warp sums runs of the row, the CTAs exchange their totals through distributed shared memory,
// and the one warp whose run holds the drawn point reads that run again and finds the token.
#include "../../include/t5_b200.h"
#include "common.cuh"

#include <cooperative_groups.h>
#include <math.h>
#include <string.h>

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxRuns = 1024;      // runs of one CTA; a run = 32 lanes x 16 bytes of the row

struct VerifyParams {
  const void *target, *draft;
  int64_t t_seq, t_row, d_seq, d_row;      // strides in elements
  const int *x, *n_draft;
  int64_t ld_x, ld_u, ld_out;
  const float *u, *u_sample;
  int *out, *accepted;
  int K, V, vec;
};

// entry of a distribution; what is not a positive finite number has no mass
__device__ __forceinline__ double mass(double r) { return r > 0.0 && r < INFINITY ? r : 0.0; }

// N consecutive values from element v (those at or behind V: 0)
template <typename T, int N>
__device__ __forceinline__ void load_run(const T* p, int v, int V, bool vec, float (&f)[N]) {
  if (vec && v + N <= V) {
    const uint4 u = *reinterpret_cast<const uint4*>(p + v);
    const T* t = reinterpret_cast<const T*>(&u);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f(t[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = v + i < V ? to_f(p[v + i]) : 0.f;
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) verify_kernel(const __grid_constant__ VerifyParams a) {
  pdl_sync();
  constexpr int N = 16 / sizeof(T), RUN = 32 * N;
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int s = blockIdx.x / cs, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  __shared__ double runs[kMaxRuns];      // sums of this CTA's runs, then their prefix sums
  __shared__ double totals[2][16];       // totals of the CTAs of the cluster, by attempt
  __shared__ double run_before;
  __shared__ int first, run_at;
  const int K = a.K, V = a.V;
  const int n = a.n_draft != nullptr ? min(max(a.n_draft[s], 0), K) : K;
  if (tid == 0) { first = n; run_at = -1; }
  __syncthreads();
  const T* tgt = reinterpret_cast<const T*>(a.target) + s * a.t_seq;
  const T* drf = a.draft != nullptr ? reinterpret_cast<const T*>(a.draft) + s * a.d_seq : nullptr;
  const int* xs = a.x + s * a.ld_x;
  for (int i = tid; i < n; i += kThreads) {
    const int x = xs[i];
    bool ok = false;
    if (x >= 0 && x < V) {
      const double p = to_f(tgt[i * a.t_row + x]), q = drf != nullptr ? to_f(drf[i * a.d_row + x]) : 1.0;
      ok = (double)a.u[s * a.ld_u + i] * q < p;
    }
    if (!ok) atomicMin(&first, i);
  }
  __syncthreads();
  const int acc = first;
  const bool refused = acc < n;
  const T* tr = tgt + acc * a.t_row;
  const T* dr = refused && drf != nullptr ? drf + acc * a.d_row : nullptr;
  const int hole = refused && drf == nullptr ? xs[acc] : -1;
  const double u = a.u_sample[s];

  // this CTA's runs: [r0, r1) of ceil(V / RUN)
  const int all = (V + RUN - 1) / RUN;
  const int r0 = (int)((int64_t)all * rank / cs), r1 = (int)((int64_t)all * (rank + 1) / cs);
  int token = -1;
  // second attempt: the refused draft equals the target everywhere it has mass, nothing is left; draw from the target
  for (int attempt = 0; attempt < 2; ++attempt) {
    const T* d = attempt == 0 ? dr : nullptr;
    const int skip = attempt == 0 ? hole : -1;
    auto values = [&](int run, double (&r)[N]) {
      const int v = run * RUN + lane * N;
      float p[N], q[N];
      load_run<T, N>(tr, v, V, a.vec, p);
      if (d != nullptr) load_run<T, N>(d, v, V, a.vec, q);
#pragma unroll
      for (int i = 0; i < N; ++i)
        r[i] = v + i == skip ? 0.0 : mass(d != nullptr ? (double)p[i] - (double)q[i] : (double)p[i]);
    };
    for (int run = r0 + w; run < r1; run += kWarps) {
      double r[N], sum = 0.0;
      values(run, r);
#pragma unroll
      for (int i = 0; i < N; ++i) sum += r[i];
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
      if (lane == 0) runs[run - r0] = sum;
    }
    __syncthreads();
    // inclusive prefix sums of the runs
    if (w == 0) {
      double carry = 0.0;
      for (int b = 0; b < r1 - r0; b += 32) {
        double v = b + lane < r1 - r0 ? runs[b + lane] : 0.0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const double y = __shfl_up_sync(0xffffffffu, v, o);
          if (lane >= o) v += y;
        }
        if (b + lane < r1 - r0) runs[b + lane] = carry + v;
        carry += __shfl_sync(0xffffffffu, v, 31);
      }
      if (lane < cs) *cluster.map_shared_rank(&totals[attempt][rank], lane) = carry;
    }
    cluster.sync();
    double before = 0.0, total = 0.0;
    int last = -1;      // the last CTA with any mass
    for (int c = 0; c < cs; ++c) {
      if (c < rank) before += totals[attempt][c];
      total += totals[attempt][c];
      if (totals[attempt][c] > 0.0) last = c;
    }
    if (!(total > 0.0)) {
      if (attempt == 0 && refused) continue;      // the same decision in every CTA of the cluster
      break;
    }
    const double t = u * total;
    // the owner: the first CTA whose runs reach beyond t (the last with mass, should rounding leave none)
    double reach = 0.0;
    int owner = last;
    for (int c = 0; c < cs; ++c) {
      reach += totals[attempt][c];
      if (reach > t) { owner = c; break; }
    }
    if (owner != rank) return;
    // the first run that reaches beyond t, else the last one with mass
    if (w == 0) {
      int at = -1;
      for (int b = 0; b < r1 - r0 && at < 0; b += 32) {
        const uint32_t hit = __ballot_sync(0xffffffffu, b + lane < r1 - r0 && before + runs[b + lane] > t);
        if (hit) at = b + __ffs(hit) - 1;
      }
      if (at < 0)
        for (at = r1 - r0 - 1; at > 0 && !(runs[at] > runs[at - 1]); --at) {}
      if (lane == 0) { run_at = at; run_before = before + (at > 0 ? runs[at - 1] : 0.0); }
    }
    __syncthreads();
    if (w != 0) return;
    double r[N], sum = 0.0;
    values(r0 + run_at, r);
#pragma unroll
    for (int i = 0; i < N; ++i) sum += r[i];
    double inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const double y = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += y;
    }
    // lane's candidates: the first of its values that reaches beyond t; the last one with mass
    double run_sum = run_before + inc - sum;
    int hit = -1, some = -1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      run_sum += r[i];
      const int v = (r0 + run_at) * RUN + lane * N + i;
      if (r[i] > 0.0) {
        if (hit < 0 && run_sum > t) hit = v;
        some = v;
      }
    }
    const uint32_t hits = __ballot_sync(0xffffffffu, hit >= 0), somes = __ballot_sync(0xffffffffu, some >= 0);
    if (hits) token = __shfl_sync(0xffffffffu, hit, __ffs(hits) - 1);
    else if (somes) token = __shfl_sync(0xffffffffu, some, 31 - __clz(somes));
    break;
  }
  // the owner's first warp, or (nothing to draw from) the first CTA
  if (token < 0 && (rank != 0 || w != 0)) return;
  int* out = a.out + s * a.ld_out;
  for (int i = lane; i <= K; i += 32) out[i] = i < acc ? xs[i] : (i == acc ? token : -1);
  if (lane == 0) a.accepted[s] = acc;
}

template <typename T>
cudaError_t run(const VerifyParams& a, int S, int cs, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(S * cs)); cfg.blockDim = dim3(kThreads); cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cs; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T>, a);
}

}  // namespace

extern "C" int t5_verify_draft(int32_t dtype, int32_t n_seqs, int32_t max_draft, int32_t vocab, const void* d_target,
                               int64_t target_seq_stride, int64_t target_row_stride, const void* d_draft,
                               int64_t draft_seq_stride, int64_t draft_row_stride, const int32_t* d_draft_tokens,
                               int64_t ld_draft_tokens, const int32_t* d_n_draft, const float* d_u_accept,
                               int64_t ld_u_accept, const float* d_u_sample, int32_t* d_out_tokens,
                               int64_t ld_out_tokens, int32_t* d_n_accepted, void* stream) {
  if (dtype != DT_F32 && dtype != DT_BF16) return T5_ERR_ARG;
  if (n_seqs < 0 || max_draft < 0 || max_draft > 1024 || vocab < 1) return T5_ERR_ARG;
  if (vocab > (1 << 20) || n_seqs > (1 << 20)) return T5_ERR_SHAPE;
  if (n_seqs == 0) return T5_OK;
  if (!d_target || !d_u_sample || !d_out_tokens || !d_n_accepted) return T5_ERR_NULL;
  if (max_draft > 0 && (!d_draft_tokens || !d_u_accept)) return T5_ERR_NULL;
  if (target_row_stride < vocab || target_seq_stride < 0 || ld_out_tokens < max_draft + 1 ||
      (max_draft > 0 && (ld_draft_tokens < max_draft || ld_u_accept < max_draft)) ||
      (d_draft != nullptr && max_draft > 0 && (draft_row_stride < vocab || draft_seq_stride < 0)))
    return T5_ERR_ARG;
  const int es = dtype == DT_F32 ? 4 : 2;
  VerifyParams a;
  memset(&a, 0, sizeof a);
  a.target = d_target; a.t_seq = target_seq_stride; a.t_row = target_row_stride;
  if (max_draft > 0) { a.draft = d_draft; a.d_seq = draft_seq_stride; a.d_row = draft_row_stride; }
  a.x = d_draft_tokens; a.ld_x = ld_draft_tokens; a.n_draft = max_draft > 0 ? d_n_draft : nullptr;
  a.u = d_u_accept; a.ld_u = ld_u_accept; a.u_sample = d_u_sample; a.out = d_out_tokens; a.ld_out = ld_out_tokens;
  a.accepted = d_n_accepted; a.K = max_draft; a.V = vocab;
  // 16-byte loads where every row starts on a 16-byte boundary, single values elsewhere
  auto even = [&](const void* p, int64_t s0, int64_t s1) {
    return ((uintptr_t)p & 15) == 0 && (s0 * es) % 16 == 0 && (s1 * es) % 16 == 0;
  };
  if (((uintptr_t)d_target % es) || ((uintptr_t)a.draft % es)) return T5_ERR_ALIGN;
  a.vec = even(d_target, a.t_seq, a.t_row) && (a.draft == nullptr || even(a.draft, a.d_seq, a.d_row));
  // eight CTAs per sequence, which the largest vocabulary also needs for its table of runs; with many sequences fewer
  const int cs = 8;
  const cudaError_t e = dtype == DT_F32 ? run<float>(a, n_seqs, cs, (cudaStream_t)stream)
                                        : run<bf16>(a, n_seqs, cs, (cudaStream_t)stream);
  return e == cudaSuccess ? T5_OK : T5_ERR_CUDA;
}
