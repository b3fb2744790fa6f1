// Appending new keys and values to a paged cache, with the rotation by position on the way.
//
// Token t of sequence s at position p: head g of k and v goes to slot p % page_size of page table[s, p / page_size].
// With rot_dim > 0 the first rot_dim columns of every head of k (and of q, if given) are rotated in pairs first:
//   (x0, x1) -> (x0 cos a - x1 sin a, x1 cos a + x0 sin a),   a = p base^(-2 i / rot_dim),  pair i = columns
//   (i, i + rot_dim / 2), or (2 i, 2 i + 1) when interleaved.
// The angle of a far position needs more than float32: p f is formed in float64 in units of whole turns
// (f = base^(-2 i / rot_dim) / 2 pi, from the host), its integer part dropped, and only the fraction (error 2^-25 turns)
// goes to the float32 sine and cosine.  One rounding to the storage type at the end.
//
// Bound: memory (each value is read once and written once).
#include "../../include/t5_b200.h"
#include "paged.cuh"

#include <math.h>

namespace {

constexpr int kMaxPairs = 64;      // rot_dim <= d_kv <= 128
constexpr int kAppendThreads = 256, kMaxTok = 8;

struct AppendParams {
  const char *k, *v;
  const char* q;
  char* q_out;
  int64_t ldq, ldk, ldv, ldqo;      // bytes
  const int *seq, *pos;
  int tokens_per_seq, n_tokens, n_seqs;
  int H, G, d_bytes;                // q heads (0: no q), kv heads, bytes of one head
  int rot_bytes, interleaved;       // bytes of one head that are rotated
  int tok;                          // tokens of a CTA
  FastDiv rot_units, per_rot;       // pairs of 16-byte chunks rotated in a head; in a token's q and k heads
  FastDiv rest, per_rest;           // chunks only copied, in a head; in a token's q and k heads
  int v_shift;                      // log2 of the chunks of a head
  FastDiv per_v;                    // chunks of a token's v
  PagedPool pool;
  int* status;
  double turns[kMaxPairs];          // base^(-2 i / rot_dim) / 2 pi
};

// A 16-byte chunk as floats and back
template <typename T> struct Chunk;
template <> struct Chunk<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void get(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <> struct Chunk<bf16> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void get(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 put(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      w[i] = *reinterpret_cast<uint32_t*>(&t);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
};

// Calls from(u) -> source, then to(u, loaded) for the CTA's share of [0, n): BATCH loads per thread are on their way
// before the first store.  gridDim.y CTAs share the items of a group of tokens.
template <int BATCH, int CHUNKS, typename From, typename To>
__device__ __forceinline__ void each_item(int n, From from, To to) {
  const int end = (int)((int64_t)n * (blockIdx.y + 1) / gridDim.y);
  for (int u = (int)((int64_t)n * blockIdx.y / gridDim.y) + threadIdx.x; u < end; u += kAppendThreads * BATCH) {
    uint4 x[BATCH][CHUNKS];
#pragma unroll
    for (int b = 0; b < BATCH; ++b)
      if (u + b * kAppendThreads < end) from(u + b * kAppendThreads, x[b]);
#pragma unroll
    for (int b = 0; b < BATCH; ++b)
      if (u + b * kAppendThreads < end) to(u + b * kAppendThreads, x[b]);
  }
}

// A CTA takes `tok` tokens: first where they go and the sines and cosines of their pairs, into shared memory, then all
// their chunks, thread by thread.  (A warp per token, with the angles in its registers, held too few loads in flight:
// 122 us on 16 prompts of up to 2048 tokens, 48 heads of 128 columns.)
template <typename T, int INTERLEAVED>
__global__ void __launch_bounds__(kAppendThreads, 5) paged_append_kernel(const __grid_constant__ AppendParams a) {
  pdl_sync();
  constexpr int N = Chunk<T>::N, BATCH = 2;
  __shared__ float2 sc[kMaxTok][kMaxPairs];
  __shared__ int64_t place[kMaxTok];      // byte offset in the pools; -1: a bad place, -2: padding
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * a.tok;
  const int nt = (int)min((int64_t)a.tok, a.n_tokens - t0);
  if (tid < nt) {
    const int pos = a.pos[t0 + tid];
    const int s = a.seq != nullptr ? a.seq[t0 + tid] : (int)((t0 + tid) / a.tokens_per_seq);
    int64_t at = -2;
    if (pos >= 0) {
      const int pi = (int)a.pool.ps.div((uint32_t)pos);
      int page = -1;
      if (s >= 0 && s < a.n_seqs && pi < a.pool.max_pages) page = a.pool.table[s * a.pool.ld_table + pi];
      at = -1;
      if (page >= 0 && page < a.pool.n_pages)
        at = page * a.pool.page_stride + (pos - pi * a.pool.page_size) * a.pool.slot_stride;
      else if (blockIdx.y == 0)
        paged_report(a.status, PAGED_BAD_APPEND);
    }
    place[tid] = at;
  }
  const int pairs = (int)a.rot_units.d * N;
  for (int i = tid; i < nt * kMaxPairs; i += kAppendThreads) {
    const int t = i / kMaxPairs, pair = i % kMaxPairs;
    if (a.rot_bytes > 0 && pair < pairs) {
      const double turn = (double)max(a.pos[t0 + t], 0) * a.turns[pair];
      sincospif(2.f * (float)(turn - rint(turn)), &sc[t][pair].x, &sc[t][pair].y);
    }
  }
  __syncthreads();
  const int H = a.H;
  // source and destination of column byte o of head h (q heads first) of the CTA's token t; NULL: none
  auto src = [&](int t, int h, int o) -> const char* {
    if (h < H) return a.q + (t0 + t) * a.ldq + h * a.d_bytes + o;
    return place[t] == -2 ? nullptr : a.k + (t0 + t) * a.ldk + (h - H) * a.d_bytes + o;
  };
  auto dst = [&](int t, int h, int o) -> char* {
    if (h < H) return a.q_out + (t0 + t) * a.ldqo + h * a.d_bytes + o;
    return place[t] < 0 ? nullptr : a.pool.k + place[t] + (h - H) * a.pool.head_stride + o;
  };
  const int second = INTERLEAVED ? 16 : a.rot_bytes / 2;      // from a unit's first chunk to its second
  if (a.rot_bytes > 0) {
    struct Unit { int t, h, c; };
    auto unit = [&](int u) {
      Unit x;
      x.t = (int)a.per_rot.div(u);
      const int r = u - x.t * (int)a.per_rot.d;
      x.h = (int)a.rot_units.div(r);
      x.c = r - x.h * (int)a.rot_units.d;
      return x;
    };
    each_item<BATCH, 2>(nt * (int)a.per_rot.d, [&](int u, uint4 (&x)[2]) {
      const Unit i = unit(u);
      const char* p = src(i.t, i.h, i.c * (INTERLEAVED ? 32 : 16));
      if (p != nullptr) {
        x[0] = *reinterpret_cast<const uint4*>(p);
        x[1] = *reinterpret_cast<const uint4*>(p + second);
      }
    }, [&](int u, const uint4 (&x)[2]) {
      const Unit i = unit(u);
      char* p = dst(i.t, i.h, i.c * (INTERLEAVED ? 32 : 16));
      if (p == nullptr) return;
      float f[2 * N], y[2 * N];
      Chunk<T>::get(x[0], f);
      Chunk<T>::get(x[1], f + N);
#pragma unroll
      for (int e = 0; e < N; ++e) {      // pair e of the unit: entries e and e + N, or 2 e and 2 e + 1
        const int lo = INTERLEAVED ? 2 * e : e, hi = INTERLEAVED ? 2 * e + 1 : e + N;
        const float2 t = sc[i.t][i.c * N + e];
        y[lo] = f[lo] * t.y - f[hi] * t.x;
        y[hi] = f[hi] * t.y + f[lo] * t.x;
      }
      *reinterpret_cast<uint4*>(p) = Chunk<T>::put(y);
      *reinterpret_cast<uint4*>(p + second) = Chunk<T>::put(y + N);
    });
  }
  // columns that are only copied: the rest of the q and k heads, and all of v
  if (a.rest.d > 0) {
    each_item<2 * BATCH, 1>(nt * (int)a.per_rest.d, [&](int u, uint4 (&x)[1]) {
      const int t = (int)a.per_rest.div(u), r = u - t * (int)a.per_rest.d, h = (int)a.rest.div(r);
      const char* p = src(t, h, a.rot_bytes + (r - h * (int)a.rest.d) * 16);
      if (p != nullptr) x[0] = *reinterpret_cast<const uint4*>(p);
    }, [&](int u, const uint4 (&x)[1]) {
      const int t = (int)a.per_rest.div(u), r = u - t * (int)a.per_rest.d, h = (int)a.rest.div(r);
      char* p = dst(t, h, a.rot_bytes + (r - h * (int)a.rest.d) * 16);
      if (p != nullptr) *reinterpret_cast<uint4*>(p) = x[0];
    });
  }
  each_item<2 * BATCH, 1>(nt * (int)a.per_v.d, [&](int u, uint4 (&x)[1]) {
    const int t = (int)a.per_v.div(u), r = u - t * (int)a.per_v.d;
    if (place[t] != -2) x[0] = *reinterpret_cast<const uint4*>(a.v + (t0 + t) * a.ldv + r * 16);
  }, [&](int u, const uint4 (&x)[1]) {
    const int t = (int)a.per_v.div(u), r = u - t * (int)a.per_v.d, h = r >> a.v_shift;
    if (place[t] >= 0)
      *reinterpret_cast<uint4*>(a.pool.v + place[t] + h * a.pool.head_stride + (r - (h << a.v_shift)) * 16) = x[0];
  });
}

template <typename T>
cudaError_t run_append(const AppendParams& a, dim3 grid, cudaStream_t st) {
  return a.interleaved ? launch_pdl(paged_append_kernel<T, 1>, grid, dim3(kAppendThreads), 0, st, a)
                       : launch_pdl(paged_append_kernel<T, 0>, grid, dim3(kAppendThreads), 0, st, a);
}

}  // namespace

cudaError_t launch_paged_append(const PagedAppendArgs& g, cudaStream_t st) {
  if (g.n_tokens == 0) return cudaSuccess;
  const int es = g.dtype == DT_F32 ? 4 : 2;
  AppendParams a;
  memset(&a, 0, sizeof a);
  a.q = (const char*)g.q; a.k = (const char*)g.k; a.v = (const char*)g.v; a.q_out = (char*)g.q_out;
  a.ldq = g.ldq * es; a.ldk = g.ldk * es; a.ldv = g.ldv * es; a.ldqo = g.ldqo * es;
  a.seq = g.seq; a.pos = g.pos; a.tokens_per_seq = g.tokens_per_seq; a.n_tokens = g.n_tokens; a.n_seqs = g.n_seqs;
  a.H = g.q != nullptr ? g.n_heads : 0; a.G = g.n_kv_heads; a.d_bytes = g.d_kv * es;
  a.rot_bytes = g.rot_dim * es; a.interleaved = g.interleaved; a.pool = g.pool; a.status = g.status;
  for (int i = 0; i < g.rot_dim / 2; ++i)
    a.turns[i] = pow(g.rot_base, -2.0 * i / g.rot_dim) / (2.0 * M_PI);
  const int heads = a.H + a.G, units = a.rot_bytes / 32, rest = (a.d_bytes - a.rot_bytes) / 16;
  a.rot_units = FastDiv(units); a.per_rot = FastDiv(heads * units);
  a.rest = FastDiv(rest); a.per_rest = FastDiv(heads * rest);
  a.per_v = FastDiv(a.G * a.d_bytes / 16);
  while ((16 << a.v_shift) < a.d_bytes) ++a.v_shift;
  // many tokens: up to kMaxTok of them in a CTA, as long as there are eight CTAs per SM.  Few: a CTA each, and several
  // CTAs share one until there are two per SM or 256 chunks for each.  (kMaxTok 1 / 4 / 8 / 16: 189 / 117 / 112 / 118 us on the
  // prompts above.)
  const int64_t chunks = (int64_t)(a.H + 2 * a.G) * a.d_bytes / 16;
  a.tok = g.n_tokens / (148 * 8);
  a.tok = a.tok < 1 ? 1 : a.tok > kMaxTok ? kMaxTok : a.tok;
  const int64_t groups = (g.n_tokens + a.tok - 1) / a.tok;
  int64_t parts = (2 * 148 + groups - 1) / groups;
  if (parts > (chunks + 255) / 256) parts = (chunks + 255) / 256;
  const dim3 grid((unsigned)groups, (unsigned)(parts < 1 ? 1 : parts));
  return g.dtype == DT_F32 ? run_append<float>(a, grid, st) : run_append<bf16>(a, grid, st);
}

int paged_pool_args(int es, int n_kv_heads, int d_kv, const void* k_pages, const void* v_pages, int n_pages, int page_size,
                    int64_t page_stride, int64_t slot_stride, int64_t head_stride, const int* table, int n_seqs,
                    int max_pages, int64_t ld_table, PagedPool* out) {
  if (!k_pages || !v_pages || !table) return T5_ERR_NULL;
  if (n_pages < 1 || page_size < 1 || n_seqs < 1 || max_pages < 1 || n_kv_heads < 1) return T5_ERR_ARG;
  if (d_kv != 32 && d_kv != 64 && d_kv != 128) return T5_ERR_ARG;
  if (ld_table < max_pages || page_stride < d_kv || slot_stride < d_kv || head_stride < d_kv) return T5_ERR_ARG;
  if ((int64_t)max_pages * page_size > (1 << 30)) return T5_ERR_SHAPE;      // positions and their tiles are 32-bit
  if (!paged_aligned(k_pages) || !paged_aligned(v_pages) || (page_stride * es) % 16 || (slot_stride * es) % 16 ||
      (head_stride * es) % 16)
    return T5_ERR_ALIGN;
  out->k = (char*)k_pages; out->v = (char*)v_pages;
  out->n_pages = n_pages; out->page_size = page_size;
  out->page_stride = page_stride * es; out->slot_stride = slot_stride * es; out->head_stride = head_stride * es;
  out->table = table; out->ld_table = ld_table; out->max_pages = max_pages;
  out->ps = FastDiv((uint32_t)page_size);
  return T5_OK;
}

extern "C" int t5_paged_kv_append(int32_t dtype, int32_t n_tokens, int32_t n_heads, int32_t n_kv_heads, int32_t d_kv,
                                  const void* d_q, int64_t ldq, const void* d_k, int64_t ldk, const void* d_v, int64_t ldv,
                                  void* d_q_out, int64_t ldqo, const int32_t* d_seq, const int32_t* d_positions,
                                  int32_t rot_dim, double rot_base, int32_t rot_interleaved, void* d_k_pages,
                                  void* d_v_pages, int32_t n_pages, int32_t page_size, int64_t page_stride,
                                  int64_t slot_stride, int64_t head_stride, const int32_t* d_page_table, int32_t n_seqs,
                                  int32_t max_pages, int64_t ld_table, void* stream) {
  if (dtype != DT_F32 && dtype != DT_BF16) return T5_ERR_ARG;
  if (n_tokens == 0) return T5_OK;
  const int es = dtype == DT_F32 ? 4 : 2;
  PagedAppendArgs a;
  memset(&a, 0, sizeof a);
  int rc = paged_pool_args(es, n_kv_heads, d_kv, d_k_pages, d_v_pages, n_pages, page_size, page_stride, slot_stride,
                           head_stride, d_page_table, n_seqs, max_pages, ld_table, &a.pool);
  if (rc != T5_OK) return rc;
  if (n_tokens < 0 || n_kv_heads > 4096) return T5_ERR_ARG;
  if (rot_dim < 0 || rot_dim > d_kv || rot_dim % 16 || (rot_interleaved != 0 && rot_interleaved != 1)) return T5_ERR_ARG;
  if (rot_dim > 0 && !(rot_base > 0.0 && rot_base < 1e300)) return T5_ERR_ARG;
  if ((d_q == nullptr) != (d_q_out == nullptr)) return T5_ERR_NULL;
  if (!d_k || !d_v || !d_seq || !d_positions) return T5_ERR_NULL;
  if (d_q != nullptr && (n_heads < 1 || n_heads > 4096 || ldq < (int64_t)n_heads * d_kv || ldqo < (int64_t)n_heads * d_kv))
    return T5_ERR_ARG;
  if (ldk < (int64_t)n_kv_heads * d_kv || ldv < (int64_t)n_kv_heads * d_kv) return T5_ERR_ARG;
  if (!paged_aligned(d_q) || !paged_aligned(d_k) || !paged_aligned(d_v) || !paged_aligned(d_q_out) || (ldk * es) % 16 ||
      (ldv * es) % 16 || (d_q != nullptr && ((ldq * es) % 16 || (ldqo * es) % 16)))
    return T5_ERR_ALIGN;
  a.dtype = dtype; a.n_tokens = n_tokens; a.n_heads = n_heads; a.n_kv_heads = n_kv_heads; a.d_kv = d_kv;
  a.q = d_q; a.k = d_k; a.v = d_v; a.q_out = d_q_out; a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldqo = ldqo;
  a.seq = d_seq; a.pos = d_positions; a.tokens_per_seq = 1; a.rot_dim = rot_dim; a.rot_base = rot_base;
  a.interleaved = rot_interleaved; a.n_seqs = n_seqs; a.status = g_kernel_status;
  return paged_result(launch_paged_append(a, (cudaStream_t)stream));
}
