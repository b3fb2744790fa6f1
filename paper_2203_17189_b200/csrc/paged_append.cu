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

struct AppendParams {
  const char *k, *v;
  const char* q;
  char* q_out;
  int64_t ldq, ldk, ldv, ldqo;      // bytes
  const int *seq, *pos;
  int tokens_per_seq, n_tokens, n_seqs;
  int H, G, d_bytes;                // q heads (0: no q), kv heads, bytes of one head
  int rot_bytes, interleaved;       // bytes of one head that are rotated
  int parts;                        // warps that share one token
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

// One warp: `parts` warps share a token's heads.  Lane = (head, unit): a unit is the two 16-byte chunks that hold N
// pairs, the same unit in every head the lane visits, so its sines and cosines are computed once per token.
template <typename T>
__global__ void __launch_bounds__(256) paged_append_kernel(const __grid_constant__ AppendParams a) {
  pdl_sync();
  constexpr int N = Chunk<T>::N;
  const int lane = threadIdx.x & 31;
  const int64_t task = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = (int)(task / a.parts), part = (int)(task % a.parts);
  if (t >= a.n_tokens) return;
  const int pos = a.pos[t];
  const int s = a.seq != nullptr ? a.seq[t] : t / a.tokens_per_seq;
  char *kd = nullptr, *vd = nullptr;      // NULL: padding or a bad place, nothing is written
  if (pos >= 0) {
    const int pi = (int)a.pool.ps.div((uint32_t)pos);
    int page = -1;
    if (s >= 0 && s < a.n_seqs && pi < a.pool.max_pages) page = a.pool.table[s * a.pool.ld_table + pi];
    if (page >= 0 && page < a.pool.n_pages) {
      const int64_t off = page * a.pool.page_stride + (pos - pi * a.pool.page_size) * a.pool.slot_stride;
      kd = a.pool.k + off;
      vd = a.pool.v + off;
    } else if (lane == 0) {
      paged_report(a.status, PAGED_BAD_APPEND);
    }
  }
  const char* ks = a.k + t * a.ldk;
  const char* vs = a.v + t * a.ldv;
  const char* qs = a.q + t * a.ldq;
  char* qd = a.q_out + t * a.ldqo;
  const int H = a.H, G = a.G, db = a.d_bytes;
  // rotated columns of the q and k heads [0, H + G)
  if (a.rot_bytes > 0) {
    const int units = a.rot_bytes / 32, hstep = 32 / units;
    const int c = lane % units, h_lane = lane / units;
    const int o0 = a.interleaved ? c * 32 : c * 16, o1 = a.interleaved ? o0 + 16 : o0 + a.rot_bytes / 2;
    float cs[N], sn[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const double turn = (double)(pos > 0 ? pos : 0) * a.turns[c * N + i];
      sincospif(2.f * (float)(turn - rint(turn)), &sn[i], &cs[i]);
    }
    const int h0 = (int)((int64_t)(H + G) * part / a.parts), h1 = (int)((int64_t)(H + G) * (part + 1) / a.parts);
    if (h_lane < hstep) {
#pragma unroll 4
      for (int h = h0 + h_lane; h < h1; h += hstep) {
        const bool is_q = h < H;
        const char* src = is_q ? qs + (int64_t)h * db : ks + (int64_t)(h - H) * db;
        char* dst = is_q ? qd + (int64_t)h * db : kd + (h - H) * a.pool.head_stride;
        if (!is_q && kd == nullptr) continue;
        float x0[N], x1[N], y0[N], y1[N];
        Chunk<T>::get(*reinterpret_cast<const uint4*>(src + o0), x0);
        Chunk<T>::get(*reinterpret_cast<const uint4*>(src + o1), x1);
        if (a.interleaved) {
#pragma unroll
          for (int i = 0; i < N; ++i) {      // the two chunks are one run of 2 N columns: pair i = entries 2 i, 2 i + 1
            const float e = 2 * i < N ? x0[(2 * i) % N] : x1[(2 * i) % N], o = 2 * i < N ? x0[(2 * i + 1) % N] : x1[(2 * i + 1) % N];
            const float u = e * cs[i] - o * sn[i], w = o * cs[i] + e * sn[i];
            if (2 * i < N) { y0[(2 * i) % N] = u; y0[(2 * i + 1) % N] = w; } else { y1[(2 * i) % N] = u; y1[(2 * i + 1) % N] = w; }
          }
        } else {
#pragma unroll
          for (int i = 0; i < N; ++i) {
            y0[i] = x0[i] * cs[i] - x1[i] * sn[i];
            y1[i] = x1[i] * cs[i] + x0[i] * sn[i];
          }
        }
        *reinterpret_cast<uint4*>(dst + o0) = Chunk<T>::put(y0);
        *reinterpret_cast<uint4*>(dst + o1) = Chunk<T>::put(y1);
      }
    }
  }
  // columns that are only copied: the rest of the q and k heads, and all of v
  const int rest = (db - a.rot_bytes) / 16;
  if (rest > 0) {
    const int n = (H + G) * rest;
    const int u1 = (int)((int64_t)n * (part + 1) / a.parts);
#pragma unroll 4
    for (int u = (int)((int64_t)n * part / a.parts) + lane; u < u1; u += 32) {
      const int h = u / rest, o = a.rot_bytes + (u - h * rest) * 16;
      if (h < H) *reinterpret_cast<uint4*>(qd + (int64_t)h * db + o) = *reinterpret_cast<const uint4*>(qs + (int64_t)h * db + o);
      else if (kd != nullptr)
        *reinterpret_cast<uint4*>(kd + (h - H) * a.pool.head_stride + o) =
            *reinterpret_cast<const uint4*>(ks + (int64_t)(h - H) * db + o);
    }
  }
  if (vd != nullptr) {
    const int per = db / 16, n = G * per;
    const int u1 = (int)((int64_t)n * (part + 1) / a.parts);
#pragma unroll 4
    for (int u = (int)((int64_t)n * part / a.parts) + lane; u < u1; u += 32) {
      const int h = u / per, o = (u - h * per) * 16;
      *reinterpret_cast<uint4*>(vd + h * a.pool.head_stride + o) = *reinterpret_cast<const uint4*>(vs + (int64_t)h * db + o);
    }
  }
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
  // few tokens: several warps share one, until the GPU has 16 warps per SM or a warp has one chunk per lane left
  const int64_t chunks = (int64_t)(a.H + 2 * a.G) * a.d_bytes / 16;
  int64_t parts = (148 * 16 + g.n_tokens - 1) / g.n_tokens;
  if (parts > (chunks + 31) / 32) parts = (chunks + 31) / 32;
  a.parts = (int)(parts < 1 ? 1 : parts);
  const int64_t blocks = ((int64_t)g.n_tokens * a.parts + 7) / 8;
  return g.dtype == DT_F32 ? launch_pdl(paged_append_kernel<float>, dim3((unsigned)blocks), dim3(256), 0, st, a)
                           : launch_pdl(paged_append_kernel<bf16>, dim3((unsigned)blocks), dim3(256), 0, st, a);
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
  if (n_tokens == 0) return T5_OK;
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
  return launch_paged_append(a, (cudaStream_t)stream) == cudaSuccess ? T5_OK : T5_ERR_CUDA;
}
