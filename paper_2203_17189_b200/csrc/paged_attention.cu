// Attention of new tokens over a paged key / value cache.
//
//   out[r, h] = sum_{j < len_r} p_j v_j,   p = softmax_j(scale q[r, h].k_j + bias[h, len_r - 1 - j]),
//   lse[r, h] = log sum_{j < len_r} exp(scale q.k_j + bias);   a row with no key gives 0 and -inf.
// Rows r = s n_q .. s n_q + n_q - 1 belong to sequence s (several new tokens of one sequence, e.g. a draft); kv head g
// serves query heads g m .. g m + m - 1.
//
// Bound: memory (the cache is read once; 4 FLOP per cached value and query row).  So the work is cut by bytes, not by
// rows: the cache of all sequences and kv heads is one line of blocks (an "item" = one sequence, one kv head, one tile
// of query rows; a block = kBK keys of an item), and CTA c of a grid that fills the GPU takes the c-th equal share of
// that line, wherever the lengths put its ends.  A running maximum and sum per query row make one pass over the data
// enough; an item that ends inside one CTA is written at once, one that is cut leaves (maximum, sum, output) of every
// piece in the workspace and a second kernel joins them.  The shares follow from the lengths alone, so the order of all
// sums, and the result, is the same in every run.
//
// Each warp streams its own keys of a block through its own ring of shared-memory stages with 16-byte asynchronous
// copies, so the main loop has no barrier; the page of a key is looked up one stage before its copy is issued.
#include "../../include/t5_b200.h"
#include "paged.cuh"

#include <math.h>

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
constexpr int kMaxCtas = 444;      // 148 SMs, at most 3 CTAs each
constexpr float kLog2e = 1.4426950408889634f;

struct AttnParams {
  const char* q;
  char* out;
  int64_t ldq, ldo;      // bytes
  float* lse;
  const int* lens;
  const float* bias;
  int n_bias;
  float scale;
  int S, n_q, H, G, m;   // m = H / G query heads per kv head
  int tiles;             // tiles of query rows per kv head: ceil(n_q m / RT)
  int cap;               // keys a page table row can name
  PagedPool pool;
  float* part;           // [ctas][2][rows][d + 2]: output, maximum, sum of the cut pieces
  int4* meta;            // [ctas]: see Piece
  int rows;              // query rows of a slot: min(RT, n_q m)
  int* status;
};

// What CTA c left in the workspace: item of its first / last piece (-1: none) and whether that piece goes on beyond it.
//   x: item whose piece in slot 0 began in an earlier CTA (-1: none)     y: 1 if that piece goes on in the next CTA
//   z: item whose piece in slot 1 began here and goes on in the next CTA (-1: none)
// (one int4; the join reads the z of its own CTA and the x, y of those behind it)

__device__ __forceinline__ int row_len(const AttnParams& a, int r) { return min(max(a.lens[r], 0), a.cap); }
__device__ __forceinline__ int seq_len(const AttnParams& a, int s) {      // keys any row of the sequence sees
  int n = 0;
  for (int i = 0; i < a.n_q; ++i) n = max(n, row_len(a, s * a.n_q + i));
  return n;
}

__device__ __forceinline__ int64_t warp_sum64(int64_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A place on the line of blocks
struct Place {
  int s, k, blk;      // sequence, item of the sequence (kv head * tiles + tile), block of the item
  int nb, len;        // blocks of an item of this sequence, keys of the sequence
};
__device__ __forceinline__ int blocks_of(int len, int bk) { return len > bk ? (len + bk - 1) / bk : 1; }
__device__ __forceinline__ void step(const AttnParams& a, int bk, Place& p) {
  if (++p.blk < p.nb) return;
  p.blk = 0;
  if (++p.k < a.G * a.tiles) return;
  p.k = 0;
  if (++p.s < a.S) { p.len = seq_len(a, p.s); p.nb = blocks_of(p.len, bk); }
}

// This CTA's share [x0, x1) of the line and the place of x0.  Called by all threads.
__device__ void find_share(const AttnParams& a, int bk, int64_t& x0, int64_t& x1, Place& p) {
  __shared__ int64_t sums[kWarps];
  __shared__ int64_t found_prefix;
  __shared__ int found_s;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  int64_t mine = 0;      // blocks per item of this thread's sequences
  int first = 0;
  for (int s = tid; s < a.S; s += kThreads) {
    const int n = blocks_of(seq_len(a, s), bk);
    if (s == tid) first = n;
    mine += n;
  }
  const int64_t ws = warp_sum64(mine);
  if (lane == 0) sums[w] = ws;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) total += sums[i];
  const int64_t items = (int64_t)a.G * a.tiles;
  total *= items;
  const int64_t c = blockIdx.x, n = gridDim.x;
  if (total >= n) { x0 = total * c / n; x1 = total * (c + 1) / n; }
  else { x0 = min(c, total); x1 = min(c + 1, total); }      // the CTAs without work lie behind all others
  if (x0 == x1) return;
  // the sequence whose blocks hold x0: prefix(s) <= x0 / items < prefix(s + 1)
  const int64_t at = x0 / items;
  int64_t base = 0;
  for (int s0 = 0; s0 < a.S; s0 += kThreads) {
    const int s = s0 + tid;
    const int n = s >= a.S ? 0 : (s0 == 0 ? first : blocks_of(seq_len(a, s), bk));
    int64_t inc = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    __syncthreads();
    if (lane == 31) sums[w] = inc;
    __syncthreads();
    int64_t before = base + inc - n, all = base;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < w) before += sums[i];
      all += sums[i];
    }
    if (n > 0 && before <= at && at < before + n) { found_s = s; found_prefix = before; }
    base = all;
    if (at < base) break;
  }
  __syncthreads();
  p.s = found_s;
  p.len = seq_len(a, p.s);
  p.nb = blocks_of(p.len, bk);
  const int64_t in = x0 - found_prefix * items;
  p.k = (int)(in / p.nb);
  p.blk = (int)(in - (int64_t)p.k * p.nb);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Chunk position of a 16-byte chunk in a tile row of CPR chunks, so that eight rows read at one chunk index hit
// eight different bank groups
template <int CPR> __device__ __forceinline__ int swz(int row, int c) {
  return CPR >= 8 ? (c ^ (row & 7)) : (c ^ ((row >> 1) & (CPR - 1)));
}

// Offset (bytes) of key j of sequence s, head g in the pools, or -1 if there is none
__device__ __forceinline__ int64_t key_offset(const AttnParams& a, const Place& p, int j) {
  if (j >= p.len) return -1;
  const int pi = (int)a.pool.ps.div((uint32_t)j);
  const int page = a.pool.table[p.s * a.pool.ld_table + pi];
  if (page < 0 || page >= a.pool.n_pages) {
    paged_report(a.status, PAGED_BAD_PAGE);
    return -1;
  }
  return page * a.pool.page_stride + (j - pi * a.pool.page_size) * a.pool.slot_stride +
         (p.k / a.tiles) * a.pool.head_stride;
}

template <typename T> __device__ __forceinline__ void chunk_floats(const uint4& u, float* f);
template <> __device__ __forceinline__ void chunk_floats<float>(const uint4& u, float* f) {
  f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
}
template <> __device__ __forceinline__ void chunk_floats<bf16>(const uint4& u, float* f) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}

// ------------------------------------------------------------------ plain arithmetic (float32 mode)
// Warp tile of KT keys: lane = (key, part of the columns) for the scores, lane = columns for the values.
template <typename T, int DK, int RT> struct Simt {
  static constexpr int ES = sizeof(T), CPR = DK * ES / 16, N = 16 / ES;
  static constexpr int KT = 4096 / (DK * ES) < 32 ? 4096 / (DK * ES) : 32;
  static constexpr int BK = KT * kWarps;
  static constexpr int TILE = KT * DK * ES, STAGES = 3;
  static constexpr int PARTS = 32 / KT, CL = CPR / PARTS;      // lanes per key, chunks per lane
  static constexpr int VC = DK / 32;                           // output columns per lane
  static constexpr int QS = RT * DK * 4;                       // float32 query rows of a warp
  static constexpr int SMEM = kWarps * (STAGES * 2 * TILE + QS + STAGES * 4) + kWarps * RT * (DK + 2) * 4;
};

template <typename T, int DK, int RT>
__global__ void __launch_bounds__(kThreads) paged_attn_simt_kernel(const __grid_constant__ AttnParams a) {
  pdl_sync();
  using L = Simt<T, DK, RT>;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  unsigned char* ring = smem + w * (L::STAGES * 2 * L::TILE);
  float* qs = reinterpret_cast<float*>(smem + kWarps * (L::STAGES * 2 * L::TILE) + w * L::QS);
  uint32_t* vmask = reinterpret_cast<uint32_t*>(smem + kWarps * (L::STAGES * 2 * L::TILE + L::QS)) + w * L::STAGES;
  float* merge = reinterpret_cast<float*>(smem + kWarps * (L::STAGES * 2 * L::TILE + L::QS + L::STAGES * 4));
  const uint32_t ring_s = (uint32_t)__cvta_generic_to_shared(ring);

  int64_t x0, x1;
  Place cur;
  find_share(a, L::BK, x0, x1, cur);
  if (x0 == x1) {
    if (tid == 0) a.meta[blockIdx.x] = make_int4(-1, 0, -1, 0);
    return;
  }
  int4 meta = make_int4(-1, 0, -1, 0);
  Place nxt = cur;                   // runs ahead of cur by the stages in flight
  int64_t to_issue = x1 - x0;

  auto lookup = [&]() -> int64_t {
    if (to_issue <= 0 || lane >= L::KT) return -1;
    return key_offset(a, nxt, nxt.blk * L::BK + w * L::KT + lane);
  };
  auto issue = [&](int stage, int64_t off) {
    if (to_issue > 0) {
      const uint32_t ok = __ballot_sync(0xffffffffu, off >= 0);
      if (lane == 0) vmask[stage] = ok;
      const uint32_t kd = ring_s + stage * 2 * L::TILE, vd = kd + L::TILE;
      const int c = lane % L::CPR;
#pragma unroll
      for (int i = 0; i < L::KT * L::CPR / 32; ++i) {
        const int row = lane / L::CPR + i * (32 / L::CPR);
        const int64_t o = __shfl_sync(0xffffffffu, off, row);
        const uint32_t d = row * (DK * L::ES) + swz<L::CPR>(row, c) * 16;
        const int64_t src = o >= 0 ? o + c * 16 : 0;
        cp_async16(kd + d, a.pool.k + src, o >= 0);
        cp_async16(vd + d, a.pool.v + src, o >= 0);
      }
      step(a, L::BK, nxt);
      --to_issue;
    }
    cp_async_commit();
  };

  int64_t off = lookup();
#pragma unroll
  for (int i = 0; i < L::STAGES - 1; ++i) { issue(i, off); off = lookup(); }

  const int key_l = lane % L::KT, part_l = lane / L::KT;
  float m[RT], l[RT], o[RT][L::VC];
  int len[RT];
  bool starts_here = cur.blk == 0;
  bool fresh = true;
  int stage = 0;
  for (int64_t x = x0; x < x1; ++x) {
    const int r0 = (cur.k % a.tiles) * RT, nr = min(RT, a.n_q * a.m - r0);      // query rows of the item
    const int g = cur.k / a.tiles;
    if (fresh) {
      fresh = false;
      __syncwarp();
      for (int idx = lane; idx < RT * DK; idx += 32) {
        const int r = r0 + idx / DK;
        float v = 0.f;
        if (idx / DK < nr)
          v = to_f(reinterpret_cast<const T*>(a.q + (int64_t)(cur.s * a.n_q + r / a.m) * a.ldq)[(g * a.m + r % a.m) * DK + idx % DK]);
        qs[idx] = v;
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY; l[r] = 0.f;
        len[r] = r < nr ? row_len(a, cur.s * a.n_q + (r0 + r) / a.m) : 0;
#pragma unroll
        for (int c = 0; c < L::VC; ++c) o[r][c] = 0.f;
        if (r < nr && lane == 0 && a.lens[cur.s * a.n_q + (r0 + r) / a.m] > a.cap) paged_report(a.status, PAGED_BAD_LENGTH);
      }
    }
    cp_async_wait<L::STAGES - 2>();
    __syncwarp();
    issue((stage + L::STAGES - 1) % L::STAGES, off);
    off = lookup();
    const int j0 = cur.blk * L::BK + w * L::KT, j = j0 + key_l;
    const uint32_t ok = vmask[stage];
    if (ok != 0) {
      const unsigned char* kt = ring + stage * 2 * L::TILE;
      const unsigned char* vt = kt + L::TILE;
      float sc[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) sc[r] = 0.f;
#pragma unroll
      for (int c = 0; c < L::CL; ++c) {
        const int ch = part_l * L::CL + c;
        float kf[L::N];
        chunk_floats<T>(*reinterpret_cast<const uint4*>(kt + key_l * (DK * L::ES) + swz<L::CPR>(key_l, ch) * 16), kf);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if (r < nr) {
#pragma unroll
            for (int i = 0; i < L::N; i += 4) {
              const float4 q4 = *reinterpret_cast<const float4*>(qs + r * DK + ch * L::N + i);
              sc[r] = fmaf(q4.x, kf[i], sc[r]); sc[r] = fmaf(q4.y, kf[i + 1], sc[r]);
              sc[r] = fmaf(q4.z, kf[i + 2], sc[r]); sc[r] = fmaf(q4.w, kf[i + 3], sc[r]);
            }
          }
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r < nr) {
#pragma unroll
          for (int of = L::KT; of < 32; of <<= 1) sc[r] += __shfl_xor_sync(0xffffffffu, sc[r], of);
          const bool seen = ((ok >> key_l) & 1) && j < len[r];
          float s = sc[r] * a.scale;
          if (a.bias != nullptr && seen)
            s += a.bias[(int64_t)(g * a.m + (r0 + r) % a.m) * a.n_bias + max(a.n_bias - len[r] + j, 0)];
          s = seen ? s : -INFINITY;
          float mx = s;
#pragma unroll
          for (int of = 16; of > 0; of >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, of));
          mx = fmaxf(m[r], mx);
          const float ref = mx == -INFINITY ? 0.f : mx;
          const float corr = exp2f((m[r] - ref) * kLog2e);
          const float p = exp2f((s - ref) * kLog2e);
          m[r] = mx;
          l[r] = l[r] * corr + p;
          sc[r] = p;
#pragma unroll
          for (int c = 0; c < L::VC; ++c) o[r][c] *= corr;
        } else {
          sc[r] = 0.f;
        }
      }
#pragma unroll 8
      for (int kk = 0; kk < L::KT; ++kk) {
        float vf[L::VC];
        const int byte = lane * L::VC * L::ES;
        const unsigned char* at = vt + kk * (DK * L::ES) + swz<L::CPR>(kk, byte >> 4) * 16 + (byte & 15);
        struct alignas(L::VC * L::ES) Cols { T v[L::VC]; };
        const Cols cols = *reinterpret_cast<const Cols*>(at);
#pragma unroll
        for (int c = 0; c < L::VC; ++c) vf[c] = to_f(cols.v[c]);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if (r < nr) {
            const float p = __shfl_sync(0xffffffffu, sc[r], kk);
            // a key this row does not see has weight 0 and may hold anything: its value must not enter
            const bool seen = RT == 1 || j0 + kk < len[r];
#pragma unroll
            for (int c = 0; c < L::VC; ++c) o[r][c] = seen ? fmaf(p, vf[c], o[r][c]) : o[r][c];
          }
        }
      }
    }
    stage = (stage + 1) % L::STAGES;
    // end of the item or of the share: join the warps, write the rows or the piece
    const bool item_ends = cur.blk + 1 == cur.nb;
    if (item_ends || x + 1 == x1) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r < nr) {
          float lt = part_l == 0 ? l[r] : 0.f;
#pragma unroll
          for (int of = 16; of > 0; of >>= 1) lt += __shfl_xor_sync(0xffffffffu, lt, of);
          float* mg = merge + (w * RT + r) * (DK + 2);
#pragma unroll
          for (int c = 0; c < L::VC; ++c) mg[lane * L::VC + c] = o[r][c];
          if (lane == 0) { mg[DK] = m[r]; mg[DK + 1] = lt; }
        }
      }
      __syncthreads();
      const bool whole = item_ends && starts_here;
      const int item = cur.s * (a.G * a.tiles) + cur.k;
      const int slot = starts_here ? 1 : 0;
      if (!whole) {
        if (slot == 0) { meta.x = item; meta.y = item_ends ? 0 : 1; } else meta.z = item;
      }
      for (int idx = tid; idx < nr * DK; idx += kThreads) {
        const int r = idx / DK, c = idx % DK;
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) mx = fmaxf(mx, merge[(i * RT + r) * (DK + 2) + DK]);
        const float ref = mx == -INFINITY ? 0.f : mx;
        float acc = 0.f, sum = 0.f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) {
          const float* mg = merge + (i * RT + r) * (DK + 2);
          const float f = exp2f((mg[DK] - ref) * kLog2e);
          acc += f * mg[c];
          sum += f * mg[DK + 1];
        }
        if (whole) {
          const int rr = r0 + r, h = g * a.m + rr % a.m, row = cur.s * a.n_q + rr / a.m;
          reinterpret_cast<T*>(a.out + (int64_t)row * a.ldo)[h * DK + c] = from_f<T>(sum == 0.f ? 0.f : acc / sum);
          if (c == 0 && a.lse != nullptr) a.lse[(int64_t)row * a.H + h] = sum == 0.f ? -INFINITY : mx + logf(sum);
        } else {
          float* pt = a.part + (((int64_t)blockIdx.x * 2 + slot) * a.rows + r) * (DK + 2);
          pt[c] = acc;
          if (c == 0) { pt[DK] = mx; pt[DK + 1] = sum; }
        }
      }
      __syncthreads();
      fresh = true;
      starts_here = true;
    }
    step(a, L::BK, cur);
  }
  cp_async_wait<0>();
  if (tid == 0) a.meta[blockIdx.x] = meta;
}

// Joins the pieces of the item that the boundary behind CTA blockIdx.x cuts first; one CTA per boundary and query row.
template <typename T, int DK, int RT>
__global__ void __launch_bounds__(128) paged_attn_join_kernel(const __grid_constant__ AttnParams a, int ctas) {
  pdl_sync();
  const int c0 = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int item = a.meta[c0].z;
  if (item < 0) return;
  const int tile = (item % (a.G * a.tiles)) % a.tiles, g = (item % (a.G * a.tiles)) / a.tiles, s = item / (a.G * a.tiles);
  const int rr = tile * RT + r;
  if (rr >= a.n_q * a.m) return;
  // pieces: slot 1 of c0, then slot 0 of the CTAs behind it up to the one where the item ends (CTAs without work
  // lie behind all others)
  __shared__ int s_last;
  if (tid == 0) s_last = ctas - 1;
  __syncthreads();
  for (int c = c0 + 1 + tid; c < ctas; c += 128) {
    const int4 mt = a.meta[c];
    if (!(mt.x == item && mt.y == 1)) { atomicMin(&s_last, c); break; }
  }
  __syncthreads();
  const int n = s_last - c0 + 1;
  auto piece = [&](int i) {
    return a.part + (((int64_t)(c0 + i) * 2 + (i == 0 ? 1 : 0)) * a.rows + r) * (DK + 2);
  };
  // four warps take every fourth piece; a lane holds DK / 32 columns
  constexpr int VC = DK / 32;
  __shared__ float red[4][DK + 2];
  float mx = -INFINITY, sum = 0.f, acc[VC];
#pragma unroll
  for (int c = 0; c < VC; ++c) acc[c] = 0.f;
  for (int i = w; i < n; i += 4) {
    const float* pt = piece(i);
    const float pm = pt[DK], ps = pt[DK + 1];
    const float nm = fmaxf(mx, pm), ref = nm == -INFINITY ? 0.f : nm;
    const float f0 = exp2f((mx - ref) * kLog2e), f1 = exp2f((pm - ref) * kLog2e);
    sum = sum * f0 + ps * f1;
#pragma unroll
    for (int c = 0; c < VC; ++c) acc[c] = acc[c] * f0 + pt[lane * VC + c] * f1;
    mx = nm;
  }
#pragma unroll
  for (int c = 0; c < VC; ++c) red[w][lane * VC + c] = acc[c];
  if (lane == 0) { red[w][DK] = mx; red[w][DK + 1] = sum; }
  __syncthreads();
  if (tid < DK) {
    mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) mx = fmaxf(mx, red[i][DK]);
    const float ref = mx == -INFINITY ? 0.f : mx;
    float v = 0.f;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float f = exp2f((red[i][DK] - ref) * kLog2e);
      v += f * red[i][tid];
      sum += f * red[i][DK + 1];
    }
    const int h = g * a.m + rr % a.m, row = s * a.n_q + rr / a.m;
    reinterpret_cast<T*>(a.out + (int64_t)row * a.ldo)[h * DK + tid] = from_f<T>(sum == 0.f ? 0.f : v / sum);
    if (tid == 0 && a.lse != nullptr) a.lse[(int64_t)row * a.H + h] = sum == 0.f ? -INFINITY : mx + logf(sum);
  }
}

int sm_count() {
  static int cached[64];
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
  if (cached[dev] == 0) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 1) n = 148;
    cached[dev] = n;
  }
  return cached[dev];
}

// Rows of one tile
int row_tile(int rows) { return rows == 1 ? 1 : 8; }

template <typename T, int DK, int RT>
cudaError_t run_simt(AttnParams& a, cudaStream_t st) {
  using L = Simt<T, DK, RT>;
  static bool set[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!set[dev]) {
    e = cudaFuncSetAttribute(paged_attn_simt_kernel<T, DK, RT>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::SMEM);
    if (e != cudaSuccess) return e;
    set[dev] = true;
  }
  int occ = 227 * 1024 / (L::SMEM + 1024);
  occ = occ > 3 ? 3 : (occ < 1 ? 1 : occ);
  int ctas = sm_count() * occ;
  if (ctas > kMaxCtas) ctas = kMaxCtas;
  a.tiles = (a.n_q * a.m + RT - 1) / RT;
  a.rows = a.n_q * a.m < RT ? a.n_q * a.m : RT;
  e = launch_pdl(paged_attn_simt_kernel<T, DK, RT>, dim3(ctas), dim3(kThreads), (size_t)L::SMEM, st, a);
  if (e != cudaSuccess) return e;
  return launch_pdl(paged_attn_join_kernel<T, DK, RT>, dim3(ctas - 1, a.rows), dim3(128), 0, st, a, ctas);
}

}  // namespace

int64_t paged_attention_workspace(int n_rows, int n_q, int H, int Hkv, int d_kv) {
  (void)n_rows;
  const int64_t all = (int64_t)n_q * (H / Hkv), rows = all < 16 ? all : 16;
  return kMaxCtas * (int64_t)sizeof(int4) + kMaxCtas * 2 * rows * (d_kv + 2) * 4;
}

cudaError_t launch_paged_attention(const PagedAttnArgs& g, cudaStream_t st) {
  if (g.n_rows == 0) return cudaSuccess;
  const int es = g.dtype == DT_F32 ? 4 : 2;
  AttnParams a;
  memset(&a, 0, sizeof a);
  a.q = (const char*)g.q; a.out = (char*)g.out; a.ldq = g.ldq * es; a.ldo = g.ldo * es; a.lse = g.lse; a.lens = g.lens;
  a.bias = g.bias; a.n_bias = g.n_bias; a.scale = g.scale;
  a.S = g.n_rows / g.n_q; a.n_q = g.n_q; a.H = g.H; a.G = g.Hkv; a.m = g.H / g.Hkv;
  a.cap = g.pool.max_pages * g.pool.page_size;
  a.pool = g.pool; a.status = g.status;
  a.meta = (int4*)g.workspace;
  a.part = (float*)((char*)g.workspace + kMaxCtas * sizeof(int4));
  const int rt = row_tile(a.n_q * a.m);
#define RUN(T, DK) (rt == 1 ? run_simt<T, DK, 1>(a, st) : run_simt<T, DK, 8>(a, st))
  if (g.dtype == DT_F32) return g.d_kv == 32 ? RUN(float, 32) : g.d_kv == 64 ? RUN(float, 64) : RUN(float, 128);
  return g.d_kv == 32 ? RUN(bf16, 32) : g.d_kv == 64 ? RUN(bf16, 64) : RUN(bf16, 128);
#undef RUN
}

extern "C" {

static int attention_shape(int32_t n_rows, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t d_kv) {
  if (n_rows < 0 || n_q < 1 || n_q > 64 || n_rows % n_q || n_heads < 1 || n_heads > 4096 || n_kv_heads < 1 ||
      n_heads % n_kv_heads)
    return T5_ERR_ARG;
  if (d_kv != 32 && d_kv != 64 && d_kv != 128) return T5_ERR_ARG;
  if ((int64_t)n_rows * n_heads > INT32_MAX / 64) return T5_ERR_SHAPE;      // item numbers are 32-bit
  return T5_OK;
}

int t5_paged_attention_workspace_bytes(int32_t n_rows, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t d_kv,
                                       int64_t* bytes) {
  if (!bytes) return T5_ERR_NULL;
  const int rc = attention_shape(n_rows, n_q, n_heads, n_kv_heads, d_kv);
  if (rc != T5_OK) return rc;
  *bytes = paged_attention_workspace(n_rows, n_q, n_heads, n_kv_heads, d_kv);
  return T5_OK;
}

int t5_paged_attention(int32_t dtype, int32_t n_rows, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t d_kv,
                       float scale, const void* d_q, int64_t ldq, const void* d_k_pages, const void* d_v_pages,
                       int32_t n_pages, int32_t page_size, int64_t page_stride, int64_t slot_stride, int64_t head_stride,
                       const int32_t* d_page_table, int32_t max_pages, int64_t ld_table, const int32_t* d_lens,
                       const float* d_bias, int32_t n_bias, void* d_out, int64_t ldo, float* d_lse, void* d_workspace,
                       int64_t workspace_bytes, void* stream) {
  if (dtype != DT_F32 && dtype != DT_BF16) return T5_ERR_ARG;
  const int es = dtype == DT_F32 ? 4 : 2;
  int rc = attention_shape(n_rows, n_q, n_heads, n_kv_heads, d_kv);
  if (rc != T5_OK) return rc;
  PagedAttnArgs a;
  memset(&a, 0, sizeof a);
  rc = paged_pool_args(es, n_kv_heads, d_kv, d_k_pages, d_v_pages, n_pages, page_size, page_stride, slot_stride, head_stride,
                       d_page_table, n_rows > 0 ? n_rows / n_q : 1, max_pages, ld_table, &a.pool);
  if (rc != T5_OK) return rc;
  if ((d_bias != nullptr) != (n_bias > 0) || n_bias < 0 || !isfinite(scale)) return T5_ERR_ARG;
  if (n_rows == 0) return T5_OK;
  if (!d_q || !d_lens || !d_out || !d_workspace) return T5_ERR_NULL;
  if (ldq < (int64_t)n_heads * d_kv || ldo < (int64_t)n_heads * d_kv) return T5_ERR_ARG;
  if (!paged_aligned(d_q) || !paged_aligned(d_out) || !paged_aligned(d_workspace) || (ldq * es) % 16 || (ldo * es) % 16)
    return T5_ERR_ALIGN;
  if (workspace_bytes < paged_attention_workspace(n_rows, n_q, n_heads, n_kv_heads, d_kv)) return T5_ERR_WORKSPACE;
  a.dtype = dtype; a.n_rows = n_rows; a.n_q = n_q; a.H = n_heads; a.Hkv = n_kv_heads; a.d_kv = d_kv;
  a.q = d_q; a.out = d_out; a.ldq = ldq; a.ldo = ldo; a.lse = d_lse; a.lens = d_lens; a.bias = d_bias; a.n_bias = n_bias;
  a.scale = scale; a.workspace = d_workspace; a.status = g_kernel_status;
  return launch_paged_attention(a, (cudaStream_t)stream) == cudaSuccess ? T5_OK : T5_ERR_CUDA;
}

}  // extern "C"
