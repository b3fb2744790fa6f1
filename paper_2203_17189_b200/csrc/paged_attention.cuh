// What the kernels of attention over a paged cache share: the line of key tiles and its shares, the query rows of an item,
// the pieces of items that are cut, and the kernel that joins those of several CTAs.
#pragma once
#include "../../include/t5_b200.h"
#include "paged.cuh"

#include <limits.h>
#include <math.h>

#include <atomic>

namespace {

constexpr int kWarps = 4, kThreads = kWarps * 32;
// CTAs of a grid at most: 148 SMs, two CTAs each (their rings take 96 KB), four with the smaller rings of narrow heads
constexpr int max_ctas(int d_kv) { return 148 * (d_kv <= 32 ? 4 : 2); }
constexpr float kLog2e = 1.4426950408889634f;
template <int DK> constexpr int kRowOf = DK + 4;      // floats of a piece's row: output, maximum, sum, two unused (16-byte rows)

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
  FastDiv by_m, by_tiles, by_items, by_workers;      // divisions by m, tiles, the items of a sequence (G tiles), the warps
  int cap;               // keys a page table row can name
  PagedPool pool;
  int runs;              // 1: pages hold whole runs of keys (KeyStream)
  float* warp_part;      // [workers][2][rows][d + 4]: output, maximum, sum of the pieces a warp leaves
  float* part;           // [ctas][2][rows][d + 4]: the same of a CTA
  int4* meta;            // [ctas]: which pieces those are, see below
  int cluster;           // CTAs per item when every item has a cluster of its own
  int extra;             // tiles that an item counts beside its own (find_share)
  int rows;              // query rows of a slot: min(RT, n_q m)
  int* status;
};

// What a share (of a warp, of a CTA) leaves of the items it cuts:
//   x: item whose piece in slot 0 began in an earlier share (-1: none)   y: 1 if that item goes on in the next share
//   z: item whose piece in slot 1 began here and goes on in the next share (-1: none)

// 2^x, results below 2^-126 as zero (they are weights relative to the largest one)
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
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

// Barrier of the CTA's first kThreads threads
__device__ __forceinline__ void sync_first() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); }

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

// This warp's share, tiles [x0, x1) of the line, and the place of x0.  Called by the CTA's first kThreads threads.
// An item counts as its tiles and a.extra more, for what its start and end cost (measured: shares of equal tiles alone ended
// 15 us apart on 128 short sequences with a bias): the line that is cut is made of such units, the extra ones in front of
// an item's tiles, and a cut inside them falls on the item's first tile.
__device__ void find_share(const AttnParams& a, int bk, int64_t& x0, int64_t& x1, Place& p) {
  constexpr int kEnds = kWarps + 1;      // where the warps' shares begin, and the next CTA's
  __shared__ int64_t sums[kWarps];
  __shared__ int64_t found_prefix[kEnds];
  __shared__ int found_s[kEnds];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  int64_t mine = 0;      // units per item of this thread's sequences
  int first = 0;
  for (int s = tid; s < a.S; s += kThreads) {
    const int n = blocks_of(seq_len(a, s), bk) + a.extra;
    if (s == tid) first = n;
    mine += n;
    if (blockIdx.x == 0)
      for (int i = 0; i < a.n_q; ++i)
        if (a.lens[s * a.n_q + i] > a.cap) paged_report(a.status, PAGED_BAD_LENGTH);
  }
  const int64_t ws = warp_sum64(mine);
  if (lane == 0) sums[w] = ws;
  sync_first();
  int64_t total = 0;
#pragma unroll
  for (int i = 0; i < kWarps; ++i) total += sums[i];
  const int64_t items = (int64_t)a.G * a.tiles, n_w = (int64_t)gridDim.x * kWarps, line = total * items;
  // Lane i looks at the CTA's i-th cut: cut c of n_w at c q + min(c, r), line = q n_w + r.  A division of 64 bits takes as
  // long as a memory access and is left to huge totals.
  const bool small = line < (1ll << 31);
  const int64_t q = small ? (int64_t)a.by_workers.div((uint32_t)line) : line / n_w, rest = line - q * n_w;
  const int64_t c = (int64_t)blockIdx.x * kWarps + min(lane, kWarps);
  const int64_t cut = c * q + min(c, rest);
  const int64_t my_at = small ? (int64_t)a.by_items.div((uint32_t)cut) : cut / items;
  int64_t at[kEnds];      // in units of one item per sequence
#pragma unroll
  for (int i = 0; i < kEnds; ++i) at[i] = __shfl_sync(0xffffffffu, my_at, i);
  // the sequences that hold the cuts: prefix(s) <= at < prefix(s + 1)
  int64_t base = 0;
  for (int s0 = 0; s0 < a.S && base <= at[kWarps]; s0 += kThreads) {
    const int s = s0 + tid;
    const int n = s >= a.S ? 0 : (s0 == 0 ? first : blocks_of(seq_len(a, s), bk) + a.extra);
    int64_t inc = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += v;
    }
    sync_first();
    if (lane == 31) sums[w] = inc;
    sync_first();
    int64_t before = base + inc - n;
#pragma unroll
    for (int i = 0; i < kWarps; ++i) {
      if (i < w) before += sums[i];
      base += sums[i];
    }
#pragma unroll
    for (int i = 0; i < kEnds; ++i)
      if (at[i] >= before && at[i] < before + n) { found_s[i] = s; found_prefix[i] = before; }
  }
  sync_first();
  // lane i: place of cut i, and the tiles in front of it
  Place m = {};
  int64_t tiles = (total - (int64_t)a.extra * a.S) * items;      // a cut at the line's end
  const int e = min(lane, kWarps);
  if (cut < line) {
    m.s = found_s[e];
    m.len = seq_len(a, m.s);
    m.nb = blocks_of(m.len, bk);
    const int64_t in = cut - found_prefix[e] * items;
    const int per = m.nb + a.extra;
    m.k = small ? (int)((uint32_t)in / (uint32_t)per) : (int)(in / per);
    m.blk = max((int)(in - (int64_t)m.k * per) - a.extra, 0);
    tiles = (found_prefix[e] - (int64_t)a.extra * m.s) * items + (int64_t)m.k * m.nb + m.blk;
  }
  x0 = __shfl_sync(0xffffffffu, tiles, w);
  x1 = __shfl_sync(0xffffffffu, tiles, w + 1);
  p.s = __shfl_sync(0xffffffffu, m.s, w); p.k = __shfl_sync(0xffffffffu, m.k, w); p.blk = __shfl_sync(0xffffffffu, m.blk, w);
  p.nb = __shfl_sync(0xffffffffu, m.nb, w); p.len = __shfl_sync(0xffffffffu, m.len, w);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(ok ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Entry of the page table for key j of the place's sequence; kNoKey where the sequence has no such key
constexpr int kNoKey = INT_MIN;
__device__ __forceinline__ int page_entry(const AttnParams& a, const Place& p, int j) {
  return j < p.len ? a.pool.table[p.s * a.pool.ld_table + a.pool.ps.div((uint32_t)j)] : kNoKey;
}
// The page it names, or -1 if there is none
__device__ __forceinline__ int page_of(const AttnParams& a, int entry) {
  if (entry >= 0 && entry < a.pool.n_pages) return entry;
  if (entry != kNoKey) paged_report(a.status, PAGED_BAD_PAGE);
  return -1;
}
// Offset (bytes) of key j of the place's sequence and head in the pools, or -1 if there is none
__device__ __forceinline__ int64_t key_offset(const AttnParams& a, const Place& p, int j) {
  const int page = page_of(a, page_entry(a, p, j)), pi = (int)a.pool.ps.div((uint32_t)j);
  if (page < 0) return -1;
  return page * a.pool.page_stride + (j - pi * a.pool.page_size) * a.pool.slot_stride +
         a.by_tiles.div(p.k) * a.pool.head_stride;
}

// The query rows of an item and what is known of them
struct Rows {
  int r0, n, g;      // first row of the tile, rows in it, kv head
  __device__ __forceinline__ Rows(const AttnParams& a, const Place& p, int rt) {
    g = (int)a.by_tiles.div(p.k);
    r0 = (p.k - g * a.tiles) * rt;
    n = min(rt, a.n_q * a.m - r0);
  }
  // row of q and query head of row r of the tile
  __device__ __forceinline__ void place(const AttnParams& a, const Place& p, int r, int& row, int& h) const {
    const int t = (int)a.by_m.div(r0 + r);
    row = p.s * a.n_q + t;
    h = g * a.m + (r0 + r - t * a.m);
  }
};

// Bookkeeping of a walk over a share: which piece an item's end leaves where
struct Pieces {
  int4 meta = make_int4(-1, 0, -1, 0);
  bool starts_here = true;
  __device__ __forceinline__ bool whole(bool item_ends) const { return item_ends && starts_here; }
  __device__ __forceinline__ int slot() const { return starts_here ? 1 : 0; }
  __device__ __forceinline__ void note(const AttnParams& a, const Place& p, bool item_ends) {
    const int item = p.s * (a.G * a.tiles) + p.k;
    if (!whole(item_ends)) {
      if (starts_here) meta.z = item;
      else { meta.x = item; meta.y = item_ends ? 0 : 1; }
    }
    starts_here = true;
  }
};

// Where the rows of an item go
__device__ __forceinline__ Place item_place(const AttnParams& a, int item) {
  Place p;
  p.s = (int)a.by_items.div(item); p.k = item - p.s * (a.G * a.tiles); p.blk = p.nb = p.len = 0;
  return p;
}
template <typename T, int DK>
__device__ __forceinline__ T* out_row(const AttnParams& a, int row, int h) {
  return reinterpret_cast<T*>(a.out + (int64_t)row * a.ldo) + h * DK;
}
__device__ __forceinline__ void write_lse(const AttnParams& a, int row, int h, float mx, float sum) {
  if (a.lse != nullptr) a.lse[(int64_t)row * a.H + h] = sum == 0.f ? -INFINITY : mx + logf(sum);
}

// two floats as bfloat16 parts: hi = round(x), lo = round(x - hi)
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(x, y);
  hi = *reinterpret_cast<const uint32_t*>(&h);
  const float2 f = __bfloat1622float2(h);
  const __nv_bfloat162 l = __floats2bfloat162_rn(x - f.x, y - f.y);
  lo = *reinterpret_cast<const uint32_t*>(&l);
}

__device__ __forceinline__ bool not_finite(uint32_t two) {      // either bfloat16 has an exponent of all ones
  return (two & 0x7f80u) == 0x7f80u || (two & 0x7f800000u) == 0x7f800000u;
}
// Joins the pieces of the item that the boundary behind CTA blockIdx.x is the first to cut, kJoinWarps query rows in a CTA.
// Up to eight pieces: a warp per row (a CTA per row took 28 us for 64 rows at 295 boundaries, 9 us for 8).  More: the warps
// take every kJoinWarps-th piece of a row, eight at a time with all their loads on the way at once, and combine what they have
// in shared memory (74 pieces, one sequence of 46,900 keys: 11 us with separate passes for maxima, sums and columns, 7 us so).
constexpr int kJoinWarps = 4;
template <typename T, int DK, int RT>
__global__ void __launch_bounds__(kJoinWarps * 32) paged_attn_join_kernel(const __grid_constant__ AttnParams a, int ctas) {
  pdl_sync();
  const int c0 = blockIdx.x, r0 = blockIdx.y * kJoinWarps, tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int item = a.meta[c0].z;
  // pieces: slot 1 of c0, then slot 0 of the CTAs behind it up to the one where the item ends (a CTA without work lies
  // between items, never inside one)
  int4 mt = a.meta[min(c0 + 1 + lane, ctas - 1)];
  if (item < 0) return;
  int last = ctas - 1;
  for (int c = c0 + 1; c < ctas; c += 32) {      // every warp looks for itself
    if (c > c0 + 1) mt = a.meta[min(c + lane, ctas - 1)];
    const uint32_t ends = __ballot_sync(0xffffffffu, c + lane < ctas && !(mt.x == item && mt.y == 1));
    if (ends) { last = c + __ffs(ends) - 1; break; }
  }
  const Place p = item_place(a, item);
  const Rows rows(a, p, RT);
  const int n = last - c0 + 1;
  constexpr int VC = DK / 32;
  struct alignas(VC * 4) Cols { float v[VC]; };
  // pieces i0, i0 + by, ... of row r: their maximum, and sum and columns relative to it
  auto gather = [&](int r, int i0, int by, float& mx, float& sum, float (&acc)[VC]) {
    mx = -INFINITY; sum = 0.f;
#pragma unroll
    for (int c = 0; c < VC; ++c) acc[c] = 0.f;
    for (; i0 < n; i0 += 8 * by) {
      float2 ms[8];      // maximum and sum
      Cols v[8];
      float top = mx;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int i = i0 + k * by;
        ms[k] = make_float2(-INFINITY, 0.f);
#pragma unroll
        for (int c = 0; c < VC; ++c) v[k].v[c] = 0.f;
        if (i < n) {
          const float* q = a.part + (((int64_t)(c0 + i) * 2 + (i == 0 ? 1 : 0)) * a.rows + r) * kRowOf<DK>;
          ms[k] = *reinterpret_cast<const float2*>(q + DK);
          v[k] = *reinterpret_cast<const Cols*>(q + lane * VC);
        }
      }
#pragma unroll
      for (int k = 0; k < 8; ++k) top = fmaxf(top, ms[k].x);
      const float ref = top == -INFINITY ? 0.f : top;
      const float f = ex2((mx - ref) * kLog2e);
      mx = top;
      sum *= f;
#pragma unroll
      for (int c = 0; c < VC; ++c) acc[c] *= f;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float e = ex2((ms[k].x - ref) * kLog2e);
        sum += e * ms[k].y;
#pragma unroll
        for (int c = 0; c < VC; ++c) acc[c] += e * v[k].v[c];
      }
    }
  };
  float mx, sum, acc[VC];
  int row, h;
  if (n <= 8) {
    if (r0 + w >= rows.n) return;
    gather(r0 + w, 0, 1, mx, sum, acc);
    rows.place(a, p, r0 + w, row, h);
#pragma unroll
    for (int c = 0; c < VC; ++c) out_row<T, DK>(a, row, h)[lane * VC + c] = from_f<T>(sum == 0.f ? 0.f : acc[c] / sum);
    if (lane == 0) write_lse(a, row, h, mx, sum);
    return;
  }
  __shared__ float red[kJoinWarps][DK], red_m[kJoinWarps], red_s[kJoinWarps];
  for (int r = r0; r < min(r0 + kJoinWarps, rows.n); ++r) {
    gather(r, w, kJoinWarps, mx, sum, acc);
#pragma unroll
    for (int c = 0; c < VC; ++c) red[w][lane * VC + c] = acc[c];
    if (lane == 0) { red_m[w] = mx; red_s[w] = sum; }
    __syncthreads();
    if (tid < DK) {
      mx = red_m[0];
#pragma unroll
      for (int i = 1; i < kJoinWarps; ++i) mx = fmaxf(mx, red_m[i]);
      const float ref = mx == -INFINITY ? 0.f : mx;
      float out = 0.f;
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < kJoinWarps; ++i) {
        const float e = ex2((red_m[i] - ref) * kLog2e);
        out += e * red[i][tid];
        sum += e * red_s[i];
      }
      rows.place(a, p, r, row, h);
      out_row<T, DK>(a, row, h)[tid] = from_f<T>(sum == 0.f ? 0.f : out / sum);
      if (tid == 0) write_lse(a, row, h, mx, sum);
    }
    __syncthreads();
  }
}

// Rows of q and new tokens that share a kv head, at most this many: the widest tile of each kernel
constexpr int kMmaRows = 16, kTcRows = 128;

inline AttnParams attn_params(const PagedAttnArgs& g) {
  const int es = g.dtype == DT_F32 ? 4 : 2;
  AttnParams a;
  memset(&a, 0, sizeof a);
  a.q = (const char*)g.q; a.out = (char*)g.out; a.ldq = g.ldq * es; a.ldo = g.ldo * es; a.lse = g.lse; a.lens = g.lens;
  a.bias = g.bias; a.n_bias = g.n_bias; a.scale = g.scale;
  a.S = g.n_rows / g.n_q; a.n_q = g.n_q; a.H = g.H; a.G = g.Hkv; a.m = g.H / g.Hkv;
  a.cap = g.pool.max_pages * g.pool.page_size;
  a.pool = g.pool; a.status = g.status;
  a.meta = (int4*)g.workspace;
  a.part = (float*)((char*)g.workspace + max_ctas(g.d_kv) * sizeof(int4));
  return a;
}
// Query rows in tiles of rt
inline void set_tiles(AttnParams& a, int rt) {
  a.tiles = (a.n_q * a.m + rt - 1) / rt;
  a.rows = a.n_q * a.m < rt ? a.n_q * a.m : rt;
  a.by_m = FastDiv(a.m); a.by_tiles = FastDiv(a.tiles); a.by_items = FastDiv(a.G * a.tiles);
}

using Kernel = void (*)(AttnParams);

// CTAs that fill the GPU with this kernel, looked up (and its shared memory allowed) once per device
template <typename T, int DK, int RT, bool CLUSTER>
cudaError_t grid_of(Kernel kernel, int smem, int* ctas) {
  static std::atomic<int> known[64];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  int n = known[dev].load(std::memory_order_acquire);
  if (n == 0) {
    int sms = 0, per_sm = 0;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, kThreads, smem);
    if (e != cudaSuccess) return e;
    n = sms * per_sm < max_ctas(DK) ? sms * per_sm : max_ctas(DK);
    if (n < 2) n = 2;
    known[dev].store(n, std::memory_order_release);
  }
  *ctas = n;
  return cudaSuccess;
}
template <typename T, int DK, int RT> cudaError_t launch_join(const AttnParams& a, int ctas, cudaStream_t st) {
  return launch_pdl(paged_attn_join_kernel<T, DK, RT>, dim3(ctas - 1, (a.rows + kJoinWarps - 1) / kJoinWarps),
                    dim3(kJoinWarps * 32), 0, st, a, ctas);
}
// The kernel over equal shares of the line, and the one that joins what it cut
template <typename T, int DK, int RT>
cudaError_t launch_line(AttnParams& a, Kernel line, int smem, cudaStream_t st) {
  int ctas = 0;
  cudaError_t e = grid_of<T, DK, RT, false>(line, smem, &ctas);
  if (e != cudaSuccess) return e;
  a.by_workers = FastDiv(ctas * kWarps);
  a.extra = a.bias != nullptr ? 2 : 1;
  e = launch_pdl(line, dim3(ctas), dim3(kThreads), (size_t)smem, st, a);
  if (e != cudaSuccess) return e;
  return launch_join<T, DK, RT>(a, ctas, st);
}

}  // namespace
