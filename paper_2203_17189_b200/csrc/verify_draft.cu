// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Sequence s has n drafted tokens x_0 .. x_{n-1}, drawn from draft_0 .. draft_{n-1} (or, without draft probabilities,
// given with certainty: draft_i is one at x_i and zero elsewhere).  x_i is accepted while u_i draft_i(x_i) < target_i(x_i),
// i.e. with probability min(1, target / draft).  Behind the a accepted tokens one more is drawn: from
// max(target_a - draft_a, 0) when x_a was refused, from target_n when none was.  The tokens then follow the target's
// distribution.  The draw inverts the cumulative sum: the first v with sum_{i <= v} r_i > u sum_i r_i.
//
// A float32 sum of 10^5 probabilities is off by enough to move the drawn point over a border, so sums carry about 48 bits:
// u draft < target is decided in float64, where the product of two float32 values is exact; differences and the sums of a
// lane are kept as two float32 parts (error-free transformations: the rounding error of a + b is itself a float32 and
// is added up beside the sum); everything behind that is float64.  (Float64 from the start cost 19.2 instead of 11.6 us on
// 256 bfloat16 rows of 32128: conversions and float64 comparisons of every value.)
//
// Bound: latency.  Only the row behind the last accepted token is read, once: 2 V values per sequence.  A cluster of CTAs
// takes one sequence; every warp sums runs of the row, the CTAs exchange their totals through distributed shared memory,
// and the one warp whose run holds the drawn point reads that run again and finds the token.
#include "../../include/t5_b200.h"
#include "paged.cuh"

#include <cooperative_groups.h>
#include <math.h>
#include <string.h>

namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxRuns = 2048;      // runs of one CTA; a run = LN values of each of a warp's lanes

struct VerifyParams {
  const void *target, *draft;
  int64_t t_seq, t_row, d_seq, d_row;      // strides in elements
  const int *x, *n_draft;
  int64_t ld_x, ld_u, ld_out;
  const float *u, *u_sample;
  int *out, *accepted;
  int K, V, vec;
};

// a sum in two parts: hi the rounded sum, lo what the roundings lost
struct Sum2 {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float x, float x_lo) {
    const float t = hi + x, b = t - hi;
    lo += ((hi - (t - b)) + (x - b)) + x_lo;
    hi = t;
  }
  __device__ __forceinline__ double value() const { return (double)hi + (double)lo; }
};
// max(p - q, 0) in two parts; what is not a positive finite number has no mass
template <bool DIFF>
__device__ __forceinline__ void mass(float p, float q, float& hi, float& lo) {
  float h = p, l = 0.f;
  if (DIFF) {
    h = p - q;
    const float b = h - p;
    l = (p - (h - b)) - (q + b);
  }
  const bool some = __float_as_uint(h) - 1u < 0x7f7fffffu;      // 0 < h < infinity
  hi = some ? h : 0.f;
  lo = DIFF && some ? l : 0.f;
}

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

// What the lanes of a warp hold of a run: chunk c of a lane = elements run * 32 LN + c * 32 N + lane * N ... of the row
template <typename T, int LN> struct RunOf {
  static constexpr int N = 16 / sizeof(T), NC = LN / N, SIZE = 32 * LN;
  float hi[LN], lo[LN];
  template <bool DIFF>
  __device__ __forceinline__ void load(const T* p, const T* q, int run, int V, bool vec, int hole, int lane) {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int v = run * SIZE + c * 32 * N + lane * N;
      float pf[N], qf[N];
      load_run<T, N>(p, v, V, vec, pf);
      if (DIFF) load_run<T, N>(q, v, V, vec, qf);
      if (hole >= v && hole < v + N) {
#pragma unroll
        for (int i = 0; i < N; ++i) pf[i] = v + i == hole ? 0.f : pf[i];
      }
#pragma unroll
      for (int i = 0; i < N; ++i) mass<DIFF>(pf[i], DIFF ? qf[i] : 0.f, hi[c * N + i], lo[c * N + i]);
    }
  }
  __device__ __forceinline__ void get(const T* p, const T* q, int run, int V, bool vec, int hole, int lane) {
    if (q != nullptr) load<true>(p, q, run, V, vec, hole, lane);
    else load<false>(p, q, run, V, vec, hole, lane);
  }
};

// Sums of this warp's runs (run w, w + kWarps, ... of [0, n)) into shared memory
template <typename T, int LN, bool DIFF>
__device__ __forceinline__ void sum_runs(const T* p, const T* q, int r0, int n, int V, bool vec, int hole, double* runs) {
  const int lane = threadIdx.x & 31;
#pragma unroll 2
  for (int run = threadIdx.x >> 5; run < n; run += kWarps) {
    RunOf<T, LN> r;
    r.template load<DIFF>(p, q, r0 + run, V, vec, hole, lane);
    Sum2 even, odd;      // two chains of dependent additions instead of one
#pragma unroll
    for (int i = 0; i < LN; i += 2) { even.add(r.hi[i], r.lo[i]); odd.add(r.hi[i + 1], r.lo[i + 1]); }
    even.add(odd.hi, odd.lo);
    double sum = even.value();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) runs[run] = sum;
  }
}

template <typename T, int LN>
__global__ void __launch_bounds__(kThreads) verify_kernel(const __grid_constant__ VerifyParams a) {
  pdl_sync();
  using R = RunOf<T, LN>;
  constexpr int N = R::N, NC = R::NC;
  cg::cluster_group cluster = cg::this_cluster();
  const int cs = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
  const int s = blockIdx.x / cs, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  __shared__ double runs[kMaxRuns];      // sums of this CTA's runs, then their prefix sums
  __shared__ double totals[2][16];       // totals of the CTAs of the cluster, by attempt
  __shared__ double run_before;
  __shared__ int first, run_at;
  const int K = a.K, V = a.V;
  const int n = a.n_draft != nullptr ? min(max(a.n_draft[s], 0), K) : K;
  const double u = fmax((double)a.u_sample[s], 0.0);      // below 0 and NaN: 0, so that what it draws has mass
  if (cs > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;");      // "has started", waited for below
  if (tid == 0) { first = K; run_at = -1; }
  __syncthreads();
  const T* tgt = reinterpret_cast<const T*>(a.target) + s * a.t_seq;
  const T* drf = a.draft != nullptr ? reinterpret_cast<const T*>(a.draft) + s * a.d_seq : nullptr;
  const int* xs = a.x + s * a.ld_x;
  for (int i = tid; i < K; i += kThreads) {      // all K, so that no load waits for n
    const int x = xs[i];
    const float ui = a.u[s * a.ld_u + i];
    bool ok = false;
    if (x >= 0 && x < V) {
      const double p = to_f(tgt[i * a.t_row + x]), q = drf != nullptr ? to_f(drf[i * a.d_row + x]) : 1.0;
      ok = (double)ui * q < p;
    }
    if (!ok) atomicMin(&first, i);
  }
  __syncthreads();
  const int acc = min(first, n);
  const bool refused = acc < n;
  const T* tr = tgt + acc * a.t_row;
  const T* dr = refused && drf != nullptr ? drf + acc * a.d_row : nullptr;
  const int hole = refused && drf == nullptr ? xs[acc] : -1;

  // this CTA's runs: [r0, r1) of those of the row
  const int all = (V + R::SIZE - 1) / R::SIZE;
  const int r0 = (int)((int64_t)all * rank / cs), r1 = (int)((int64_t)all * (rank + 1) / cs);
  int token = -1;
  // second attempt: the refused draft equals the target everywhere it has mass, nothing is left; draw from the target
  for (int attempt = 0; attempt < 2; ++attempt) {
    const T* d = attempt == 0 ? dr : nullptr;
    const int skip = attempt == 0 ? hole : -1;
    if (d != nullptr) sum_runs<T, LN, true>(tr, d, r0, r1 - r0, V, a.vec, skip, runs);
    else sum_runs<T, LN, false>(tr, d, r0, r1 - r0, V, a.vec, skip, runs);
    // CTAs write to each other next: all have to have started
    if (attempt == 0 && cs > 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
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
    if (cs > 1) cluster.sync();
    else __syncthreads();
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
    R r;
    r.get(tr, d, r0 + run_at, V, a.vec, skip, lane);
    double reached = run_before;      // in front of the chunk
    int some = -1;                    // this lane's last value with mass, should rounding leave none beyond t
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      double sum = 0.0;
#pragma unroll
      for (int i = 0; i < N; ++i) sum += (double)r.hi[c * N + i] + (double)r.lo[c * N + i];
      double inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const double y = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += y;
      }
      double at = reached + inc - sum;
      int hit = -1;
#pragma unroll
      for (int i = 0; i < N; ++i) {
        at += (double)r.hi[c * N + i] + (double)r.lo[c * N + i];
        const int v = (r0 + run_at) * R::SIZE + c * 32 * N + lane * N + i;
        if (r.hi[c * N + i] > 0.f) {
          if (hit < 0 && at > t) hit = v;
          some = v;
        }
      }
      const uint32_t hits = __ballot_sync(0xffffffffu, hit >= 0);
      if (hits && token < 0) token = __shfl_sync(0xffffffffu, hit, __ffs(hits) - 1);
      reached += __shfl_sync(0xffffffffu, inc, 31);
    }
    if (token < 0) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) some = max(some, __shfl_xor_sync(0xffffffffu, some, o));
      token = some;
    }
    break;
  }
  // the owner's first warp, or (nothing to draw from) the first CTA
  if (token < 0 && (rank != 0 || w != 0)) return;
  int* out = a.out + s * a.ld_out;
  for (int i = lane; i <= K; i += 32) out[i] = i < acc ? xs[i] : (i == acc ? token : -1);
  if (lane == 0) a.accepted[s] = acc;
}

// CTAs per sequence: as many as leave every SM at most two.  Measured (vocabulary 32128, float32 with draft
// probabilities, us with 8 / 4 / 2 / 1 CTAs): 1 sequence 5.4 / 6.1 / 7.7 / 10.8, 32: 6.7 / 6.9 / 8.0 / 11.1,
// 64: 12.1 / 7.5 / 8.0 / 11.1, 148: 25.1 / 16.9 / 10.9 / 12.2, 256: 47.1 / 29.2 / 21.9 / 18.2.
template <int LN>
int cluster_size(int n_seqs, int vocab) {
  int cs = 8;
  while (cs > 1 && n_seqs * cs > 2 * 148) cs /= 2;
  while (cs < 8 && vocab > cs * kMaxRuns * 32 * LN) cs *= 2;      // a CTA's table of runs
  return cs;
}

template <typename T, int LN>
cudaError_t run(const VerifyParams& a, int S, int cs, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(S * cs)); cfg.blockDim = dim3(kThreads); cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cs; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr; cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, verify_kernel<T, LN>, a);
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
  constexpr int LN = 8;      // 16 and 32 values per lane: 14.3 and 15.9 instead of 12.2 us on 148 float32 sequences
  const int cs = cluster_size<LN>(n_seqs, vocab);
  const cudaError_t e = dtype == DT_F32 ? run<float, LN>(a, n_seqs, cs, (cudaStream_t)stream)
                                        : run<bf16, LN>(a, n_seqs, cs, (cudaStream_t)stream);
  return paged_result(e);
}
