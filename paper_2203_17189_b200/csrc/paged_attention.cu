// Attention of new tokens over a paged key / value cache.
//
//   out[r, h] = sum_{j < len_r} p_j v_j,   p = softmax_j(scale q[r, h].k_j + bias[h, len_r - 1 - j]),
//   lse[r, h] = log sum_{j < len_r} exp(scale q.k_j + bias);   a row with no key gives 0 and -inf.
// Rows r = s n_q .. s n_q + n_q - 1 belong to sequence s (several new tokens of one sequence, e.g. a draft); kv head g
// serves query heads g m .. g m + m - 1.
//
// Bound: memory (the cache is read once; 4 FLOP per cached value and query row).  So the work is cut by bytes, not by
// rows: the cache of all sequences and kv heads is one line of key tiles (an "item" = one sequence, one kv head, one tile
// of query rows; its keys in tiles of 4 KB), and warp w of a grid that fills the GPU takes the w-th equal share of that
// line, wherever the lengths put its ends.  A running maximum and sum per query row make one pass over the data enough;
// an item that lies inside one share is written at once, one that is cut leaves (output, maximum, sum) of every piece in
// the workspace: the CTA joins the pieces of its four warps, a second kernel those of several CTAs.  The shares follow
// from the lengths alone, so the order of all sums, and the result, is the same in every run.
//
// A warp streams its tiles through its own ring of shared-memory stages with 16-byte asynchronous copies that run ahead
// over the ends of items, and the page of a key is looked up one tile before its copy is issued; nothing in the main loop
// waits for another warp.  (Shares per CTA, with the four warps on the keys of one item, paid for a join at every item:
// 128 sequences of 64 - 512 keys, 32 heads of 64 columns, took 137 us.)
#include "paged_attention.cuh"

#include <cooperative_groups.h>

namespace cg = cooperative_groups;

namespace {

// Chunk position of a 16-byte chunk in a tile row of CPR chunks, so that eight rows read at one chunk index hit
// eight different bank groups
template <int CPR> __device__ __forceinline__ int swz(int row, int c) {
  return CPR >= 8 ? (c ^ (row & 7)) : (c ^ ((row >> 1) & (CPR - 1)));
}

// Shape of a warp's tiles: KT keys of DK columns of ES bytes, K then V, in a ring of STAGES.  4 KB of each where 32 lanes
// can name the keys.  A run of keys lies in one page when the page size is a multiple of it.
template <int ES, int DK> struct Tile {
  static constexpr int ROW = DK * ES, CPR = ROW / 16;
  static constexpr int KT = 4096 / ROW < 32 ? 4096 / ROW : 32;
  static constexpr int RUN = KT < 16 ? KT : 16, NR = KT / RUN;
  static constexpr int BYTES = KT * ROW, STAGES = 3;
  static constexpr int RING = STAGES * 2 * BYTES;
};

// A warp's stream of tiles: runs ahead of the arithmetic by STAGES - 1 tiles, over the ends of items.  Two ways to find
// the keys of a tile: with pages of whole runs one look-up per run, the rows behind it by their stride; otherwise one per
// key, passed between lanes.
template <typename L> struct KeyStream {
  const AttnParams& a;
  Place at;             // of the next tile to be copied
  int left;             // tiles still to be copied
  int64_t off;          // this lane's run or key of that tile: its page has been looked up one step ahead
  unsigned char* ring;
  uint32_t ring_s;
  uint32_t* vmask;      // per stage: which keys of the tile exist
  int lane;

  __device__ __forceinline__ void lookup() {
    off = -1;
    if (left > 0 && lane < (a.runs ? L::NR : L::KT)) off = key_offset(a, at, at.blk * L::KT + lane * (a.runs ? L::RUN : 1));
  }
  __device__ __forceinline__ void issue(int stage) {
    if (left > 0) {
      constexpr int RPI = 32 / L::CPR;      // rows one instruction of the warp covers
      constexpr uint32_t kAll = L::KT == 32 ? 0xffffffffu : (1u << L::KT) - 1u;
      const int c = lane % L::CPR, r0 = lane / L::CPR;
      // place of row r0 + i RPI, chunk c: the swizzle's row bits come in by one exclusive-or
      const uint32_t kd = ring_s + stage * 2 * L::BYTES + r0 * L::ROW + swz<L::CPR>(r0, c) * 16;
      auto place = [&](int i) { return (kd ^ (swz<L::CPR>(i * RPI, 0) * 16)) + i * RPI * L::ROW; };
      uint32_t ok = __ballot_sync(0xffffffffu, off >= 0);
      if (a.runs) {
        const int n = at.len - at.blk * L::KT;      // keys of the sequence from here on
        uint32_t have = 0;
#pragma unroll
        for (int i = 0; i < L::NR; ++i) have |= ((ok >> i) & 1) ? ((1u << L::RUN) - 1u) << (i * L::RUN) : 0u;
        if (n < L::KT) have &= (1u << max(n, 0)) - 1u;
        ok = have;
        const int64_t dv = (intptr_t)a.pool.v - (intptr_t)a.pool.k, dr = RPI * a.pool.slot_stride;
#pragma unroll
        for (int run = 0; run < L::NR; ++run) {
          const int64_t o = __shfl_sync(0xffffffffu, off, run);
          const char* src = a.pool.k + (o >= 0 ? o : 0) + r0 * a.pool.slot_stride + c * 16;
          if (ok == kAll) {
#pragma unroll
            for (int i = run * (L::RUN / RPI); i < (run + 1) * (L::RUN / RPI); ++i, src += dr) {
              cp_async16(place(i), src);
              cp_async16(place(i) + L::BYTES, src + dv);
            }
          } else {
#pragma unroll
            for (int i = run * (L::RUN / RPI); i < (run + 1) * (L::RUN / RPI); ++i, src += dr) {
              const bool in = (ok >> (r0 + i * RPI)) & 1;
              cp_async16(place(i), src, in);      // a key that does not exist becomes zeros
              cp_async16(place(i) + L::BYTES, src + dv, in);
            }
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < L::KT / RPI; ++i) {
          const int64_t o = __shfl_sync(0xffffffffu, off, r0 + i * RPI);
          const int64_t src = o >= 0 ? o + c * 16 : 0;
          cp_async16(place(i), a.pool.k + src, o >= 0);
          cp_async16(place(i) + L::BYTES, a.pool.v + src, o >= 0);
        }
      }
      if (lane == 0) vmask[stage] = ok;
      step(a, L::KT, at);
      --left;
    }
    cp_async_commit();
    lookup();
  }
  __device__ __forceinline__ KeyStream(const AttnParams& p, const Place& from, int64_t n, unsigned char* r, uint32_t* vm,
                                       int ln)
      : a(p), at(from), left((int)n), ring(r), ring_s((uint32_t)__cvta_generic_to_shared(r)), vmask(vm), lane(ln) {
    lookup();
#pragma unroll
    for (int i = 0; i < L::STAGES - 1; ++i) issue(i);
  }
};

// End of a CTA: joins the pieces its warps left.  A chain of them that begins and ends here is an item's rows; one that
// reaches beyond this CTA's first or last warp becomes the CTA's piece.  The rows of all chains are dealt out to the warps.
// Called by all threads.
template <typename T, int DK, int RT>
__device__ void finish_cta(const AttnParams& a, const int4& mine) {
  __shared__ int4 metas[kWarps];
  const int tid = threadIdx.x, lane = tid & 31;
  if (lane == 0) metas[tid >> 5] = mine;
  __syncthreads();      // also orders the warps' pieces in global memory before the reads below
  constexpr int VC = DK / 32;
  const int64_t piece = (int64_t)a.rows * kRowOf<DK>;
  const float* parts = a.warp_part + (int64_t)blockIdx.x * kWarps * 2 * piece;
  int4 meta = make_int4(metas[0].x, 0, -1, 0);
  int turn = 0;      // rows seen so far: warp w takes those with turn % kWarps == w
  for (int w = -1; w < kWarps; ++w) {
    // the chain that begins with warp w's slot 1, or (w = -1) with the first warp's slot 0
    const int item = w < 0 ? metas[0].x : metas[w].z;
    if (item < 0) continue;
    int end = w < 0 ? 0 : w;
    bool goes_on = w < 0 ? metas[0].y != 0 : true;
    while (goes_on && end + 1 < kWarps) goes_on = metas[++end].y != 0;
    const int n = end - w + (w < 0 ? 0 : 1);      // pieces: w < 0: slots 0 of warps 0 .. end; else slot 1 of w, slots 0 behind it
    const bool whole = w >= 0 && !goes_on;
    if (goes_on) { if (w < 0) meta.y = 1; else meta.z = item; }
    const Place p = item_place(a, item);
    const Rows rows(a, p, RT);
    const float* first = parts + (w < 0 ? 0 : 2 * w + 1) * piece;
    const int64_t second = w < 0 ? 2 * piece : piece;      // from the first piece to the one behind it; then 2 piece
#pragma unroll 4
    for (int r = ((tid >> 5) - turn) & (kWarps - 1); r < rows.n; r += kWarps) {
      float mx = -INFINITY, sum = 0.f, pm[kWarps], pl[kWarps], v[kWarps][VC], acc[VC];
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        const float* q = first + (i == 0 ? 0 : second + (i - 1) * 2 * piece) + r * kRowOf<DK>;
        pm[i] = -INFINITY; pl[i] = 0.f;
        if (i < n) { pm[i] = q[DK]; pl[i] = q[DK + 1]; }
#pragma unroll
        for (int c = 0; c < VC; ++c) v[i][c] = i < n ? q[lane + 32 * c] : 0.f;
        mx = fmaxf(mx, pm[i]);
      }
      const float ref = mx == -INFINITY ? 0.f : mx;
#pragma unroll
      for (int c = 0; c < VC; ++c) acc[c] = 0.f;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        const float e = ex2((pm[i] - ref) * kLog2e);
        sum += e * pl[i];
#pragma unroll
        for (int c = 0; c < VC; ++c) acc[c] += e * v[i][c];
      }
      if (whole) {
        int row, h;
        rows.place(a, p, r, row, h);
#pragma unroll
        for (int c = 0; c < VC; ++c) out_row<T, DK>(a, row, h)[lane + 32 * c] = from_f<T>(sum == 0.f ? 0.f : acc[c] / sum);
        if (lane == 0) write_lse(a, row, h, mx, sum);
      } else {
        float* pt = a.part + ((int64_t)blockIdx.x * 2 + (w < 0 ? 0 : 1)) * piece + r * kRowOf<DK>;
#pragma unroll
        for (int c = 0; c < VC; ++c) pt[lane + 32 * c] = acc[c];
        if (lane == 0) { pt[DK] = mx; pt[DK + 1] = sum; }
      }
    }
    turn += rows.n;
  }
  if (tid == 0) a.meta[blockIdx.x] = meta;
}

// Short caches and few items: a cluster of a.cluster CTAs per item instead of shares of the line.  Its warps take equal
// runs of the item's tiles and join through distributed shared memory, which spares the second kernel and the search.
__device__ __forceinline__ void cluster_share(const AttnParams& a, int bk, int64_t& x0, int64_t& x1, Place& p) {
  const int item = blockIdx.x / a.cluster, n = a.cluster * kWarps;
  const int w = (blockIdx.x - item * a.cluster) * kWarps + (threadIdx.x >> 5);
  p = item_place(a, item);
  p.len = seq_len(a, p.s);
  p.nb = blocks_of(p.len, bk);
  x0 = p.nb * w / n;
  x1 = p.nb * (w + 1) / n;
  p.blk = (int)x0;
  if (blockIdx.x == item * a.cluster && p.k == 0 && threadIdx.x < a.n_q && a.lens[p.s * a.n_q + threadIdx.x] > a.cap)
    paged_report(a.status, PAGED_BAD_LENGTH);
}
// Joins the warps of a cluster: warp w of each CTA has left its rows ([row][DK + 4]: output, maximum, sum) at smem + w *
// stride.  A warp of the cluster takes 32 columns of a row; lane i looks at piece i's maximum and sum.
template <typename T, int DK, int RT>
__device__ void finish_cluster(const AttnParams& a, const Place& p, unsigned char* smem, int stride) {
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  const Rows rows(a, p, RT);
  const int lane = threadIdx.x & 31, n = a.cluster * kWarps;      // at most 32 pieces
  const int rank = (int)cluster.block_rank();
  for (int unit = rank * kWarps + (threadIdx.x >> 5); unit < rows.n * (DK / 32); unit += n) {
    const int r = unit / (DK / 32), c = unit % (DK / 32) * 32 + lane;
    auto piece = [&](int i) {
      return reinterpret_cast<const float*>(cluster.map_shared_rank(smem + (i % kWarps) * stride, i / kWarps)) + r * kRowOf<DK>;
    };
    float m = -INFINITY, l = 0.f;
    if (lane < n) { m = piece(lane)[DK]; l = piece(lane)[DK + 1]; }
    float mx = m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
    const float e = ex2((m - (mx == -INFINITY ? 0.f : mx)) * kLog2e);
    float sum = e * l, acc = 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll 8
    for (int i = 0; i < n; ++i) acc += __shfl_sync(0xffffffffu, e, i) * piece(i)[c];
    int row, h;
    rows.place(a, p, r, row, h);
    out_row<T, DK>(a, row, h)[c] = from_f<T>(sum == 0.f ? 0.f : acc / sum);
    if (c == 0) write_lse(a, row, h, mx, sum);
  }
  cluster.sync();      // nobody leaves while its shared memory is read
}

// ------------------------------------------------------------------ float32: plain arithmetic
// Lane = (key, part of the columns) for the scores, lane = columns for the values.
template <int DK, int RT> struct Simt : Tile<4, DK> {
  using B = Tile<4, DK>;
  static constexpr int PARTS = 32 / B::KT, CL = B::CPR / PARTS;      // lanes per key, chunks per lane
  static constexpr int VC = DK / 32;                                 // output columns per lane
  static constexpr int QS = RT * DK * 4;                             // query rows of a warp's item
  static constexpr int PS = RT > 1 ? B::KT * RT * 4 : 0;             // weights of a tile, [key][row]
  static constexpr int SMEM = kWarps * (B::RING + QS + PS + B::STAGES * 4);
};

template <int DK, int RT, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 2) paged_attn_simt_kernel(const __grid_constant__ AttnParams a) {
  pdl_sync();
  using L = Simt<DK, RT>;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  float* qs = reinterpret_cast<float*>(smem + kWarps * L::RING + w * L::QS);
  float* ps = reinterpret_cast<float*>(smem + kWarps * (L::RING + L::QS) + w * L::PS);
  uint32_t* vmask = reinterpret_cast<uint32_t*>(smem + kWarps * (L::RING + L::QS + L::PS)) + w * L::STAGES;

  int64_t x0, x1;
  Place cur = {};
  if (CLUSTER) cluster_share(a, L::KT, x0, x1, cur);
  else find_share(a, L::KT, x0, x1, cur);
  Pieces pieces;
  pieces.starts_here = cur.blk == 0;
  float* part = a.warp_part + ((int64_t)blockIdx.x * kWarps + w) * 2 * a.rows * kRowOf<DK>;
  KeyStream<L> keys(a, cur, x1 - x0, smem + w * L::RING, vmask, lane);

  const int key_l = lane % L::KT, part_l = lane / L::KT;
  float m[RT], l[RT], o[RT][L::VC];
  int len[RT], head[RT], q_row[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) {      // a warp of a cluster may have no tile at all
    m[r] = -INFINITY; l[r] = 0.f;
#pragma unroll
    for (int c = 0; c < L::VC; ++c) o[r][c] = 0.f;
  }
  bool fresh = true;
  int stage = 0;
  for (int64_t x = x0; x < x1; ++x) {
    const Rows rows(a, cur, RT);
    const int nr = rows.n;
    if (fresh) {
      fresh = false;
      // lane r < nr looks its row up; the row's columns are then copied by all lanes
      int row = 0, h = 0, row_keys = 0;
      if (lane < nr) {
        rows.place(a, cur, lane, row, h);
        row_keys = a.n_q == 1 ? cur.len : row_len(a, row);
      }
      const int64_t at = (int64_t)row * a.ldq + (int64_t)h * DK * 4;
      __syncwarp();
      constexpr int PER = DK / 4;      // float4 of a row
#pragma unroll
      for (int i = 0; i < (RT * PER + 31) / 32; ++i) {
        const int idx = i * 32 + lane, r = idx / PER;
        const int64_t o = __shfl_sync(0xffffffffu, at, r & 31);
        if (r < RT) {      // rows beyond the tile's are zero: they see no key
          const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
          reinterpret_cast<float4*>(qs)[idx] = r < nr ? *reinterpret_cast<const float4*>(a.q + o + (idx % PER) * 16) : none;
        }
      }
      __syncwarp();
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        m[r] = -INFINITY; l[r] = 0.f;
        len[r] = __shfl_sync(0xffffffffu, row_keys, r);
        head[r] = __shfl_sync(0xffffffffu, h, r);
        q_row[r] = __shfl_sync(0xffffffffu, row, r);
#pragma unroll
        for (int c = 0; c < L::VC; ++c) o[r][c] = 0.f;
      }
    }
    cp_async_wait<L::STAGES - 2>();
    __syncwarp();
    keys.issue((stage + L::STAGES - 1) % L::STAGES);
    const int j0 = cur.blk * L::KT, j = j0 + key_l;
    const uint32_t ok = vmask[stage];
    if (ok != 0) {
      const unsigned char* kt = keys.ring + stage * 2 * L::BYTES;
      const unsigned char* vt = kt + L::BYTES;
      float sc[RT], add[RT];
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        sc[r] = add[r] = 0.f;
        if (a.bias != nullptr && j < len[r]) add[r] = a.bias[(int64_t)head[r] * a.n_bias + max(a.n_bias - len[r] + j, 0)];
      }
#pragma unroll
      for (int c = 0; c < L::CL; ++c) {
        const int ch = part_l * L::CL + c;
        const float4 k4 = *reinterpret_cast<const float4*>(kt + key_l * L::ROW + swz<L::CPR>(key_l, ch) * 16);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          const float4 q4 = *reinterpret_cast<const float4*>(qs + r * DK + ch * 4);
          sc[r] = fmaf(q4.x, k4.x, sc[r]); sc[r] = fmaf(q4.y, k4.y, sc[r]);
          sc[r] = fmaf(q4.z, k4.z, sc[r]); sc[r] = fmaf(q4.w, k4.w, sc[r]);
        }
      }
      // a tile's keys are summed by themselves and then added: KT + n / KT roundings instead of n
      float corr[RT], t[RT][L::VC];
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < L::VC; ++c) t[r][c] = 0.f;
      bool all_see = true;      // every row sees every key of the tile that exists
#pragma unroll
      for (int r = 0; r < RT; ++r) {
#pragma unroll
        for (int of = L::KT; of < 32; of <<= 1) sc[r] += __shfl_xor_sync(0xffffffffu, sc[r], of);
        const bool seen = ((ok >> key_l) & 1) && j < len[r];
        all_see &= r >= nr || min(j0 + L::KT, cur.len) <= len[r];
        const float s = seen ? fmaf(sc[r], a.scale, add[r]) : -INFINITY;
        float mx = s;
#pragma unroll
        for (int of = 16; of > 0; of >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, of));
        mx = fmaxf(m[r], mx);
        const float ref = mx == -INFINITY ? 0.f : mx;
        corr[r] = ex2((m[r] - ref) * kLog2e);
        sc[r] = ex2((s - ref) * kLog2e);
        m[r] = mx;
        l[r] = l[r] * corr[r] + sc[r];
      }
      if (RT > 1) {      // the weights in shared memory: two loads give a key's weights of eight rows
        __syncwarp();
        if (part_l == 0) {
#pragma unroll
          for (int r = 0; r < RT; ++r) ps[key_l * RT + r] = sc[r];
        }
        __syncwarp();
      }
      struct alignas(L::VC * 4) Cols { float v[L::VC]; };
      auto values = [&](int kk) {
        const int byte = lane * L::VC * 4;
        return *reinterpret_cast<const Cols*>(vt + kk * L::ROW + swz<L::CPR>(kk, byte >> 4) * 16 + (byte & 15));
      };
      if (RT == 1) {
#pragma unroll 8
        for (int kk = 0; kk < L::KT; ++kk) {
          const Cols vf = values(kk);
          const float p = __shfl_sync(0xffffffffu, sc[0], kk);
#pragma unroll
          for (int c = 0; c < L::VC; ++c) t[0][c] = fmaf(p, vf.v[c], t[0][c]);
        }
      } else if (all_see) {
#pragma unroll 8
        for (int kk = 0; kk < L::KT; ++kk) {
          const Cols vf = values(kk);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const float p = ps[kk * RT + r];
#pragma unroll
            for (int c = 0; c < L::VC; ++c) t[r][c] = fmaf(p, vf.v[c], t[r][c]);
          }
        }
      } else {
        // a key that a row does not see has weight 0 there and may hold anything: its value must not enter
#pragma unroll 1
        for (int kk = 0; kk < L::KT; ++kk) {
          const Cols vf = values(kk);
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            const float p = ps[kk * RT + r];
#pragma unroll
            for (int c = 0; c < L::VC; ++c) t[r][c] = j0 + kk < len[r] ? fmaf(p, vf.v[c], t[r][c]) : t[r][c];
          }
        }
      }
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int c = 0; c < L::VC; ++c) o[r][c] = fmaf(o[r][c], corr[r], t[r][c]);
    }
    stage = (stage + 1) % L::STAGES;
    const bool item_ends = cur.blk + 1 == cur.nb;
    if (!CLUSTER && (item_ends || x + 1 == x1)) {
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r < nr) {
          float lt = part_l == 0 ? l[r] : 0.f;
#pragma unroll
          for (int of = 16; of > 0; of >>= 1) lt += __shfl_xor_sync(0xffffffffu, lt, of);
          const bool whole = pieces.whole(item_ends);
          const int h = head[r], row = q_row[r];
          float* at = whole ? out_row<float, DK>(a, row, h) : part + (pieces.slot() * a.rows + r) * kRowOf<DK>;
#pragma unroll
          for (int c = 0; c < L::VC; ++c) at[lane * L::VC + c] = !whole ? o[r][c] : (lt == 0.f ? 0.f : o[r][c] / lt);
          if (lane == 0) {
            if (whole) write_lse(a, row, h, m[r], lt);
            else { at[DK] = m[r]; at[DK + 1] = lt; }
          }
        }
      }
      pieces.note(a, cur, item_ends);
      fresh = true;
    }
    if (CLUSTER) ++cur.blk;
    else step(a, L::KT, cur);
  }
  cp_async_wait<0>();
  if (CLUSTER) {
    __syncwarp();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      float lt = part_l == 0 ? l[r] : 0.f;
#pragma unroll
      for (int of = 16; of > 0; of >>= 1) lt += __shfl_xor_sync(0xffffffffu, lt, of);
      float* at = reinterpret_cast<float*>(keys.ring) + r * kRowOf<DK>;
#pragma unroll
      for (int c = 0; c < L::VC; ++c) at[lane * L::VC + c] = o[r][c];
      if (lane == 0) { at[DK] = m[r]; at[DK + 1] = lt; }
    }
    finish_cluster<float, DK, RT>(a, cur, smem, L::RING);
  } else {
    finish_cta<float, DK, RT>(a, pieces.meta);
  }
}

// ------------------------------------------------------------------ bfloat16: matrix instructions
// m16n8k16 products with float32 sums.  Up to 8 query rows (heads that share the kv head, new tokens of the sequence) are
// the 8 columns of S^T = K Q^T and O^T += V^T P^T, 16 keys or 16 columns the 16 rows (paged_attn_rows8_kernel): 24
// instructions per 16 keys of 128 columns.  With more rows they are the 16 rows of S = Q K^T and O += P V, 16 at a time
// (paged_attn_rows16_kernel): 48; 8 rows as half of 16 took 305 instead of 292 us on 6 x 29 heads of 64 columns over 47,600
// keys.  A single row fills an eighth of the instructions, which costs nothing more.  tcgen05 has 128 rows and a trip through
// tensor memory per tile (paged_attention_tc.cu takes it, for more than 16 rows); here neither operand nor result leaves the
// registers between load and use.  What bounds these kernels beside memory is the two warps that a scheduler has (registers and rings allow no more): about 430
// instructions per 8 KB at five cycles each.
// The weights go into the second product as a sum of two bfloat16 parts (error 2^-17 instead of 2^-9), so the output is the
// float32 result rounded once; without the second part the calls above take 0 - 5 % less.
template <int DK> struct Mma : Tile<2, DK> {
  using B = Tile<2, DK>;
  static constexpr int SMEM = kWarps * (B::RING + B::STAGES * 4);
};

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
// c += a b: c[0..1] row lane / 4, c[2..3] row lane / 4 + 8, columns 2 (lane % 4) + 0, 1
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 8 x 8 transpose of pairs: in, lane holds row lane / 4, columns 2 (lane % 4) + 0, 1
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// O += P V of one tile without a product that a row does not see: s [2 tiles of 8 keys per 16][4], o [DK / 8][4] as in the
// kernel of 16 rows; rows lane / 4 (+ 8) see the first n0 / n1 keys
template <int DK>
__device__ __noinline__ void values_by_key16(const unsigned char* vt, const float* s, float* o, int n0, int n1) {
  using L = Mma<DK>;
  const int lane = threadIdx.x & 31, quad = lane & 3;
  for (int kk = 0; kk < L::KT; ++kk)
    for (int hf = 0; hf < 2; ++hf) {
      const float p = __shfl_sync(0xffffffffu, s[(kk / 8) * 4 + 2 * hf + (kk & 1)], (lane & ~3) | ((kk & 7) >> 1));
      if (kk < (hf ? n1 : n0))
        for (int t = 0; t < DK / 8; ++t) {
          const uint32_t u = *reinterpret_cast<const uint32_t*>(vt + kk * L::ROW + swz<L::CPR>(kk, t) * 16 + quad * 4);
          o[t * 4 + 2 * hf] = fmaf(p, __uint_as_float(u << 16), o[t * 4 + 2 * hf]);
          o[t * 4 + 2 * hf + 1] = fmaf(p, __uint_as_float(u & 0xffff0000u), o[t * 4 + 2 * hf + 1]);
        }
    }
}
// The same for the kernel of 8 rows: s [16 keys][4], o [DK / 16][4]; rows 2 (lane % 4) + 0, 1 see the first n0 / n1 keys
template <int DK>
__device__ __noinline__ void values_by_key8(const unsigned char* vt, const float* s, float* o, int n0, int n1) {
  using L = Mma<DK>;
  const int lane = threadIdx.x & 31, quad = lane & 3;
  for (int kk = 0; kk < L::KT; ++kk)
    for (int j = 0; j < 2; ++j) {
      const float p = __shfl_sync(0xffffffffu, s[(kk / 16) * 4 + ((kk >> 3) & 1) * 2 + j], (kk & 7) * 4 + quad);
      if (kk < (j ? n1 : n0))
        for (int t = 0; t < DK / 8; ++t) {      // column 8 t + lane / 4
          const bf16 v = *reinterpret_cast<const bf16*>(vt + kk * L::ROW + swz<L::CPR>(kk, t) * 16 + (lane >> 2) * 2);
          o[(t / 2) * 4 + (t & 1) * 2 + j] = fmaf(p, to_f(v), o[(t / 2) * 4 + (t & 1) * 2 + j]);
        }
    }
}
template <int DK, int N>      // whether a tile of values holds one that is not finite
__device__ __forceinline__ bool tile_not_finite(const unsigned char* vt, int lane) {
  bool bad = false;
#pragma unroll
  for (int i = 0; i < N / 512; ++i) {
    const uint4 u = *reinterpret_cast<const uint4*>(vt + (i * 32 + lane) * 16);
    bad |= not_finite(u.x) | not_finite(u.y) | not_finite(u.z) | not_finite(u.w);
  }
  return __any_sync(0xffffffffu, bad);
}

template <int DK, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, max_ctas(DK) / 148) paged_attn_rows8_kernel(const __grid_constant__ AttnParams a) {
  pdl_sync();
  using L = Mma<DK>;
  constexpr int RT = 8;
  constexpr int KS = DK / 16, NG = L::KT / 16, NT = DK / 16;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, quad = lane & 3;
  uint32_t* vmask = reinterpret_cast<uint32_t*>(smem + kWarps * L::RING) + w * L::STAGES;

  int64_t x0, x1;
  Place cur = {};
  if (CLUSTER) cluster_share(a, L::KT, x0, x1, cur);
  else find_share(a, L::KT, x0, x1, cur);
  Pieces pieces;
  pieces.starts_here = cur.blk == 0;
  float* part = a.warp_part + ((int64_t)blockIdx.x * kWarps + w) * 2 * a.rows * kRowOf<DK>;
  KeyStream<L> keys(a, cur, x1 - x0, smem + w * L::RING, vmask, lane);

  uint32_t qf[KS][2];                    // B operand: columns 16 ks + 2 quad (+ 8) of row lane / 4
  // scores of this lane: keys lane / 4 + 8 (i / 2) of each 16, rows 2 quad + i % 2; outputs: columns 16 t + lane / 4 +
  // 8 (i / 2), the same rows
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f}, o[NT][4] = {}, far[2], add[NG][4] = {}, next[NG][4] = {};
  const float* bias[2];
  int len[2], min_len = 0;      // keys this lane's rows see; the fewest of any row
  bool fresh = true;
  int stage = 0;
  for (int64_t x = x0; x < x1; ++x) {
    // What is added to the scores of a tile from key j0 on.  Behind the distance where the bias saturates that is one value
    // per row.  Loads of an SM come back in the order they went out, so a tile's bias is fetched in front of the copies
    // that follow the tile's own: fetched when it is needed it cost 0.85 us a tile.
    auto load_add = [&](int j0, float (&to)[NG][4]) {
      if (a.n_bias - min_len + j0 + L::KT - 1 > 0) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int at = a.n_bias - len[j] + j0 + (lane >> 2);
#pragma unroll
          for (int g = 0; g < NG * 2; ++g) to[g / 2][(g & 1) * 2 + j] = bias[j][min(max(at + g * 8, 0), a.n_bias - 1)];
        }
      } else {
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) to[g][i] = far[i & 1];
      }
    };
    if (fresh) {
      fresh = false;
      const Rows rows(a, cur, RT);
      min_len = 0x7fffffff;
      int row, h;      // rows beyond the tile's repeat its first one and are not kept
      rows.place(a, cur, (lane >> 2) < rows.n ? lane >> 2 : 0, row, h);
      const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (int64_t)row * a.ldq + h * (DK * 2)) + quad;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qf[ks][0] = src[ks * 8];
        qf[ks][1] = src[ks * 8 + 4];
      }
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        rows.place(a, cur, quad * 2 + j < rows.n ? quad * 2 + j : 0, row, h);
        m[j] = -INFINITY; l[j] = 0.f; far[j] = 0.f; bias[j] = a.bias;
        len[j] = a.n_q == 1 ? cur.len : row_len(a, row);      // one token: known from the walk
        min_len = min(min_len, len[j]);
        if (a.bias != nullptr) { bias[j] = a.bias + (int64_t)h * a.n_bias; far[j] = bias[j][0]; }
      }
      if (a.n_q > 1) {
        min_len = min(min_len, __shfl_xor_sync(0xffffffffu, min_len, 1));
        min_len = min(min_len, __shfl_xor_sync(0xffffffffu, min_len, 2));
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[t][i] = 0.f;
      if (a.bias != nullptr) load_add(cur.blk * L::KT, add);
    }
    const int j0 = cur.blk * L::KT;
    if (a.bias != nullptr && cur.blk + 1 < cur.nb) load_add(j0 + L::KT, next);
    cp_async_wait<L::STAGES - 2>();
    __syncwarp();
    keys.issue((stage + L::STAGES - 1) % L::STAGES);
    const uint32_t ok = vmask[stage];
    if (ok != 0) {
      const uint32_t kt = keys.ring_s + stage * 2 * L::BYTES, vt = kt + L::BYTES;
      float s[NG][4];
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[g][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t b[4];
          const int row = g * 16 + (lane & 15);
          ldsm4(kt + row * L::ROW + swz<L::CPR>(row, 2 * ks + (lane >> 4)) * 16, b);
          mma16816(s[g], b, qf[ks][0], qf[ks][1]);
        }
      }
      // scores: scale, bias, mask
      const bool all_seen = ok == (L::KT == 32 ? 0xffffffffu : (1u << L::KT) - 1u) && j0 + L::KT <= min_len;
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[g][i] = fmaf(s[g][i], a.scale, add[g][i]);
      if (!all_seen) {
        const uint32_t mine = ok >> (lane >> 2);
#pragma unroll
        for (int g = 0; g < NG * 2; ++g)
#pragma unroll
          for (int j = 0; j < 2; ++j)
            if (!((mine >> (g * 8)) & 1) || j0 + g * 8 + (lane >> 2) >= len[j]) s[g / 2][(g & 1) * 2 + j] = -INFINITY;
      }
      float top[2] = {m[0], m[1]}, ref[2];
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[i & 1] = fmaxf(top[i & 1], s[g][i]);
      bool moved = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
#pragma unroll
        for (int of = 4; of < 32; of <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], of));
        ref[j] = top[j] == -INFINITY ? 0.f : top[j];
        moved |= top[j] != m[j];
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const float corr = ex2((m[j] - ref[j]) * kLog2e);
          l[j] *= corr;
          m[j] = top[j];
#pragma unroll
          for (int t = 0; t < NT; ++t) { o[t][j] *= corr; o[t][2 + j] *= corr; }
        }
      }
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[g][i] = ex2((s[g][i] - ref[i & 1]) * kLog2e);      // differences first: a bias of the lowest float stays finite
          l[i & 1] += s[g][i];
        }
      // Keys that one row sees and another does not have weight 0 there, and 0 x NaN would spoil the row: if such a tile
      // holds a value that is not finite, it is taken key by key.
      const unsigned char* values = keys.ring + stage * 2 * L::BYTES + L::BYTES;
      const bool plain = min_len < min(j0 + L::KT, cur.len) && tile_not_finite<DK, L::BYTES>(values, lane);
      if (!plain) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t hi[2], lo[2];      // weights of keys 0 - 7 and 8 - 15: from [key][row] to [row][key]
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            split2(s[g][2 * i], s[g][2 * i + 1], hi[i], lo[i]);
            hi[i] = transpose8(hi[i]);
            lo[i] = transpose8(lo[i]);
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            uint32_t b[4];
            const int row = g * 16 + (lane & 7) + (lane >> 4) * 8;
            ldsm4_t(vt + row * L::ROW + swz<L::CPR>(row, 2 * t + ((lane >> 3) & 1)) * 16, b);
            mma16816(o[t], b, hi[0], hi[1]);
            mma16816(o[t], b, lo[0], lo[1]);
          }
        }
      } else {
        // copies, so that the rare call below does not push the registers of the others into memory
        float sc[NG * 4], oc[NT * 4];
#pragma unroll
        for (int i = 0; i < NG * 4; ++i) sc[i] = s[i / 4][i % 4];
#pragma unroll
        for (int i = 0; i < NT * 4; ++i) oc[i] = o[i / 4][i % 4];
        values_by_key8<DK>(values, sc, oc, len[0] - j0, len[1] - j0);
#pragma unroll
        for (int i = 0; i < NT * 4; ++i) o[i / 4][i % 4] = oc[i];
      }
    }
    stage = (stage + 1) % L::STAGES;
    if (a.bias != nullptr) {
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) add[g][i] = next[g][i];
    }
    const bool item_ends = cur.blk + 1 == cur.nb;
    if (!CLUSTER && (item_ends || x + 1 == x1)) {
      const Rows rows(a, cur, RT);
      const bool whole = pieces.whole(item_ends);
      float lt[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        lt[j] = l[j];
#pragma unroll
        for (int of = 4; of < 32; of <<= 1) lt[j] += __shfl_xor_sync(0xffffffffu, lt[j], of);
      }
      if (whole) {
        int row, h;
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (lane < 4 && quad * 2 + j < rows.n) {
            rows.place(a, cur, quad * 2 + j, row, h);
            write_lse(a, row, h, m[j], lt[j]);
          }
        const float inv0 = lt[0] == 0.f ? 0.f : 1.f / lt[0], inv1 = lt[1] == 0.f ? 0.f : 1.f / lt[1];
        const bool mine = (lane >> 2) < rows.n;
        rows.place(a, cur, mine ? lane >> 2 : 0, row, h);
        bf16* at = out_row<bf16, DK>(a, row, h) + quad * 2;
#pragma unroll
        for (int t = 0; t < NT * 2; ++t) {      // columns 8 t ...: from [column][row] to [row][column]
          const __nv_bfloat162 v = __floats2bfloat162_rn(o[t / 2][(t & 1) * 2] * inv0, o[t / 2][(t & 1) * 2 + 1] * inv1);
          const uint32_t u = transpose8(*reinterpret_cast<const uint32_t*>(&v));
          if (mine) *reinterpret_cast<uint32_t*>(at + t * 8) = u;
        }
      } else {
#pragma unroll
        for (int j = 0; j < 2; ++j)
          if (quad * 2 + j < rows.n) {
            float* at = part + (pieces.slot() * a.rows + quad * 2 + j) * kRowOf<DK>;
#pragma unroll
            for (int t = 0; t < NT * 2; ++t) at[t * 8 + (lane >> 2)] = o[t / 2][(t & 1) * 2 + j];
            if (lane < 4) { at[DK] = m[j]; at[DK + 1] = lt[j]; }
          }
      }
      pieces.note(a, cur, item_ends);
      fresh = true;
    }
    if (CLUSTER) ++cur.blk;
    else step(a, L::KT, cur);
  }
  cp_async_wait<0>();
  if (CLUSTER) {
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float lt = l[j];
#pragma unroll
      for (int of = 4; of < 32; of <<= 1) lt += __shfl_xor_sync(0xffffffffu, lt, of);
      float* at = reinterpret_cast<float*>(keys.ring) + (quad * 2 + j) * kRowOf<DK>;
#pragma unroll
      for (int t = 0; t < NT * 2; ++t) at[t * 8 + (lane >> 2)] = o[t / 2][(t & 1) * 2 + j];
      if (lane < 4) { at[DK] = m[j]; at[DK + 1] = lt; }
    }
    finish_cluster<bf16, DK, RT>(a, cur, smem, L::RING);
  } else {
    finish_cta<bf16, DK, RT>(a, pieces.meta);
  }
}

template <int DK, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, max_ctas(DK) / 148) paged_attn_rows16_kernel(const __grid_constant__ AttnParams a) {
  pdl_sync();
  using L = Mma<DK>;
  constexpr int RT = 16, NH = 2;         // row halves: this lane's rows are lane / 4 (+ 8)
  constexpr int KS = DK / 16, NG = L::KT / 16, NT = DK / 8, CN = 4;
  extern __shared__ __align__(128) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5, quad = lane & 3;
  uint32_t* vmask = reinterpret_cast<uint32_t*>(smem + kWarps * L::RING) + w * L::STAGES;

  int64_t x0, x1;
  Place cur = {};
  if (CLUSTER) cluster_share(a, L::KT, x0, x1, cur);
  else find_share(a, L::KT, x0, x1, cur);
  Pieces pieces;
  pieces.starts_here = cur.blk == 0;
  float* part = a.warp_part + ((int64_t)blockIdx.x * kWarps + w) * 2 * a.rows * kRowOf<DK>;
  KeyStream<L> keys(a, cur, x1 - x0, smem + w * L::RING, vmask, lane);

  uint32_t qf[KS][4];                    // A operand: columns 16 ks + 2 quad (+ 8), rows lane / 4 (+ 8)
  float m[NH], l[NH], o[NT][CN], far[NH], add[NG * 2][CN] = {}, next[NG * 2][CN] = {};
  const float* bias[NH];
  int len[NH], min_len = 0;      // keys this lane's rows see; the fewest of any row
#pragma unroll
  for (int hf = 0; hf < NH; ++hf) { m[hf] = -INFINITY; l[hf] = 0.f; }      // a warp of a cluster may have no tile at all
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int i = 0; i < CN; ++i) o[t][i] = 0.f;
  bool fresh = true;
  int stage = 0;
  for (int64_t x = x0; x < x1; ++x) {
    // What is added to the scores of a tile from key j0 on.  Behind the distance where the bias saturates that is one value
    // per row.  Loads of an SM come back in the order they went out, so a tile's bias is fetched in front of the copies
    // that follow the tile's own: fetched when it is needed it cost 0.85 us a tile.
    auto load_add = [&](int j0, float (&to)[NG * 2][CN]) {
      if (a.n_bias - min_len + j0 + L::KT - 1 > 0) {
#pragma unroll
        for (int hf = 0; hf < NH; ++hf) {
          const int at = a.n_bias - len[hf] + j0 + quad * 2;
#pragma unroll
          for (int t = 0; t < NG * 2; ++t)
#pragma unroll
            for (int i = 0; i < 2; ++i) to[t][2 * hf + i] = bias[hf][min(max(at + t * 8 + i, 0), a.n_bias - 1)];
        }
      } else {
#pragma unroll
        for (int t = 0; t < NG * 2; ++t)
#pragma unroll
          for (int i = 0; i < CN; ++i) to[t][i] = far[i >> 1];
      }
    };
    if (fresh) {
      fresh = false;
      const Rows rows(a, cur, RT);
      min_len = 0x7fffffff;
#pragma unroll
      for (int hf = 0; hf < NH; ++hf) {
        const int r = lane / 4 + 8 * hf;
        const bool valid = r < rows.n;      // rows beyond the tile's repeat its first one and are not kept
        int row, h;
        rows.place(a, cur, valid ? r : 0, row, h);
        m[hf] = -INFINITY; l[hf] = 0.f; far[hf] = 0.f; bias[hf] = a.bias;
        len[hf] = a.n_q == 1 ? cur.len : row_len(a, row);      // one token: known from the walk
        min_len = min(min_len, len[hf]);
        if (a.bias != nullptr) { bias[hf] = a.bias + (int64_t)h * a.n_bias; far[hf] = bias[hf][0]; }
        const uint32_t* src = reinterpret_cast<const uint32_t*>(a.q + (int64_t)row * a.ldq + h * (DK * 2)) + quad;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
          qf[ks][hf] = src[ks * 8];
          qf[ks][NH + hf] = src[ks * 8 + 4];
        }
      }
      if (a.n_q > 1) {
#pragma unroll
        for (int of = 4; of < 32; of <<= 1) min_len = min(min_len, __shfl_xor_sync(0xffffffffu, min_len, of));
      }
#pragma unroll
      for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int i = 0; i < CN; ++i) o[t][i] = 0.f;
      if (a.bias != nullptr) load_add(cur.blk * L::KT, add);
    }
    const int j0 = cur.blk * L::KT;
    if (a.bias != nullptr && cur.blk + 1 < cur.nb) load_add(j0 + L::KT, next);
    cp_async_wait<L::STAGES - 2>();
    __syncwarp();
    keys.issue((stage + L::STAGES - 1) % L::STAGES);
    const uint32_t ok = vmask[stage];
    if (ok != 0) {
      const uint32_t kt = keys.ring_s + stage * 2 * L::BYTES, vt = kt + L::BYTES;
      float s[NG * 2][CN];
#pragma unroll
      for (int t = 0; t < NG * 2; ++t)
#pragma unroll
        for (int i = 0; i < CN; ++i) s[t][i] = 0.f;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t b[4];
          const int row = g * 16 + (lane & 7) + ((lane >> 4) & 1) * 8;
          ldsm4(kt + row * L::ROW + swz<L::CPR>(row, 2 * ks + ((lane >> 3) & 1)) * 16, b);
          mma16816(s[2 * g], qf[ks], b[0], b[1]);
          mma16816(s[2 * g + 1], qf[ks], b[2], b[3]);
        }
      }
      // scores: scale, bias, mask
      const bool all_seen = ok == (L::KT == 32 ? 0xffffffffu : (1u << L::KT) - 1u) && j0 + L::KT <= min_len;
      float top[NH];
#pragma unroll
      for (int hf = 0; hf < NH; ++hf) top[hf] = m[hf];
#pragma unroll
      for (int t = 0; t < NG * 2; ++t)
#pragma unroll
        for (int i = 0; i < CN; ++i) s[t][i] = fmaf(s[t][i], a.scale, add[t][i]);
      if (!all_seen) {
        const uint32_t mine = ok >> (quad * 2);
#pragma unroll
        for (int t = 0; t < NG * 2; ++t)
#pragma unroll
          for (int i = 0; i < CN; ++i)
            if (!((mine >> (t * 8 + (i & 1))) & 1) || j0 + t * 8 + quad * 2 + (i & 1) >= len[i >> 1]) s[t][i] = -INFINITY;
      }
#pragma unroll
      for (int t = 0; t < NG * 2; ++t)
#pragma unroll
        for (int i = 0; i < CN; ++i) top[i >> 1] = fmaxf(top[i >> 1], s[t][i]);
      float ref[NH];
      bool moved = false;
#pragma unroll
      for (int hf = 0; hf < NH; ++hf) {
        top[hf] = fmaxf(top[hf], __shfl_xor_sync(0xffffffffu, top[hf], 1));
        top[hf] = fmaxf(top[hf], __shfl_xor_sync(0xffffffffu, top[hf], 2));
        ref[hf] = top[hf] == -INFINITY ? 0.f : top[hf];
        moved |= top[hf] != m[hf];
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int hf = 0; hf < NH; ++hf) {
          const float corr = ex2((m[hf] - ref[hf]) * kLog2e);
          l[hf] *= corr;
          m[hf] = top[hf];
#pragma unroll
          for (int t = 0; t < NT; ++t) { o[t][2 * hf] *= corr; o[t][2 * hf + 1] *= corr; }
        }
      }
#pragma unroll
      for (int t = 0; t < NG * 2; ++t)
#pragma unroll
        for (int i = 0; i < CN; ++i) {
          const int hf = i >> 1;
          s[t][i] = ex2((s[t][i] - ref[hf]) * kLog2e);      // differences first: a bias of the lowest float stays finite
          l[hf] += s[t][i];
        }
      // Keys that one row sees and another does not have weight 0 there, and 0 x NaN would spoil the row: if such a tile
      // holds a value that is not finite, it is taken key by key.
      const unsigned char* values = keys.ring + stage * 2 * L::BYTES + L::BYTES;
      const bool plain = min_len < min(j0 + L::KT, cur.len) && tile_not_finite<DK, L::BYTES>(values, lane);
      if (!plain) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) split2(s[2 * g + i / 2][2 * (i & 1)], s[2 * g + i / 2][2 * (i & 1) + 1], hi[i], lo[i]);
#pragma unroll
          for (int t = 0; t < NT; t += 2) {
            uint32_t b[4];
            const int row = g * 16 + (lane & 7) + ((lane >> 3) & 1) * 8;
            ldsm4_t(vt + row * L::ROW + swz<L::CPR>(row, t + ((lane >> 4) & 1)) * 16, b);
            mma16816(o[t], hi, b[0], b[1]);
            mma16816(o[t + 1], hi, b[2], b[3]);
            mma16816(o[t], lo, b[0], b[1]);
            mma16816(o[t + 1], lo, b[2], b[3]);
          }
        }
      } else {
        // copies, so that the rare call below does not push the registers of the others into memory
        float sc[NG * 2 * CN], oc[NT * CN];
#pragma unroll
        for (int i = 0; i < NG * 2 * CN; ++i) sc[i] = s[i / CN][i % CN];
#pragma unroll
        for (int i = 0; i < NT * CN; ++i) oc[i] = o[i / CN][i % CN];
        values_by_key16<DK>(values, sc, oc, len[0] - j0, len[1] - j0);
#pragma unroll
        for (int i = 0; i < NT * CN; ++i) o[i / CN][i % CN] = oc[i];
      }
    }
    stage = (stage + 1) % L::STAGES;
    if (a.bias != nullptr) {
#pragma unroll
      for (int t = 0; t < NG * 2; ++t)
#pragma unroll
        for (int i = 0; i < CN; ++i) add[t][i] = next[t][i];
    }
    const bool item_ends = cur.blk + 1 == cur.nb;
    if (!CLUSTER && (item_ends || x + 1 == x1)) {
      const Rows rows(a, cur, RT);
      const bool whole = pieces.whole(item_ends);
#pragma unroll
      for (int hf = 0; hf < NH; ++hf) {
        float lt = l[hf];
        lt += __shfl_xor_sync(0xffffffffu, lt, 1);
        lt += __shfl_xor_sync(0xffffffffu, lt, 2);
        const int r = lane / 4 + 8 * hf;
        if (r < rows.n) {
          if (whole) {
            int row, h;
            rows.place(a, cur, r, row, h);
            bf16* at = out_row<bf16, DK>(a, row, h) + quad * 2;
            const float inv = lt == 0.f ? 0.f : 1.f / lt;
#pragma unroll
            for (int t = 0; t < NT; ++t)
              *reinterpret_cast<__nv_bfloat162*>(at + t * 8) = __floats2bfloat162_rn(o[t][2 * hf] * inv, o[t][2 * hf + 1] * inv);
            if (quad == 0) write_lse(a, row, h, m[hf], lt);
          } else {
            float* at = part + (pieces.slot() * a.rows + r) * kRowOf<DK>;
#pragma unroll
            for (int t = 0; t < NT; ++t)
              *reinterpret_cast<float2*>(at + t * 8 + quad * 2) = make_float2(o[t][2 * hf], o[t][2 * hf + 1]);
            if (quad == 0) { at[DK] = m[hf]; at[DK + 1] = lt; }
          }
        }
      }
      pieces.note(a, cur, item_ends);
      fresh = true;
    }
    if (CLUSTER) ++cur.blk;
    else step(a, L::KT, cur);
  }
  cp_async_wait<0>();
  if (CLUSTER) {
    __syncwarp();
#pragma unroll
    for (int hf = 0; hf < NH; ++hf) {
      float lt = l[hf];
      lt += __shfl_xor_sync(0xffffffffu, lt, 1);
      lt += __shfl_xor_sync(0xffffffffu, lt, 2);
      float* at = reinterpret_cast<float*>(keys.ring) + (lane / 4 + 8 * hf) * kRowOf<DK>;
#pragma unroll
      for (int t = 0; t < NT; ++t)
        *reinterpret_cast<float2*>(at + t * 8 + quad * 2) = make_float2(o[t][2 * hf], o[t][2 * hf + 1]);
      if (quad == 0) { at[DK] = m[hf]; at[DK + 1] = lt; }
    }
    finish_cluster<bf16, DK, RT>(a, cur, smem, L::RING);
  } else {
    finish_cta<bf16, DK, RT>(a, pieces.meta);
  }
}

// A cluster per item when all clusters are resident at once and no warp gets more than four tiles, by the keys the page
// table could name; 0: shares of the line
int cluster_size(int64_t items, int64_t cap, int kt) {
  const int64_t tiles = (cap + kt - 1) / kt;
  int c = 1;
  while (c < 8 && c * kWarps < tiles) c *= 2;
  return items * c <= 2 * 148 && tiles <= 4 * c * kWarps ? c : 0;
}

template <typename T, int DK, int RT>
cudaError_t run_attention(AttnParams& a, Kernel line, Kernel clustered, int smem, cudaStream_t st) {
  using L = Tile<sizeof(T), DK>;
  a.runs = a.pool.page_size % L::RUN == 0;
  set_tiles(a, RT);
  const int64_t items = (int64_t)a.S * a.G * a.tiles;
  a.cluster = cluster_size(items, a.cap, L::KT);
  if (a.cluster > 0) {
    int ctas = 0;
    cudaError_t e = grid_of<T, DK, RT, true>(clustered, smem, &ctas);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(items * a.cluster)); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = a.cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, clustered, a);
  }
  return launch_line<T, DK, RT>(a, line, smem, st);
}
// Rows of a tile: the float32 kernel's arithmetic goes with them (1, 4, 8), the matrix kernels take 8 or 16
template <int DK, int RT> cudaError_t run_simt(AttnParams& a, cudaStream_t st) {
  return run_attention<float, DK, RT>(a, paged_attn_simt_kernel<DK, RT, false>, paged_attn_simt_kernel<DK, RT, true>, Simt<DK, RT>::SMEM, st);
}
template <int DK> cudaError_t run_f32(AttnParams& a, cudaStream_t st) {
  const int rows = a.n_q * a.m;
  return rows == 1 ? run_simt<DK, 1>(a, st) : rows <= 4 ? run_simt<DK, 4>(a, st) : run_simt<DK, 8>(a, st);
}
template <int DK> cudaError_t run_bf16(AttnParams& a, cudaStream_t st) {
  if (a.n_q * a.m <= 8)
    return run_attention<bf16, DK, 8>(a, paged_attn_rows8_kernel<DK, false>, paged_attn_rows8_kernel<DK, true>, Mma<DK>::SMEM, st);
  return run_attention<bf16, DK, 16>(a, paged_attn_rows16_kernel<DK, false>, paged_attn_rows16_kernel<DK, true>, Mma<DK>::SMEM, st);
}

}  // namespace

int64_t paged_attention_workspace(int n_rows, int n_q, int H, int Hkv, int d_kv) {
  (void)n_rows;
  const int64_t all = (int64_t)n_q * (H / Hkv), ctas = max_ctas(d_kv);
  // pieces of each CTA and its warps, or of a CTA of the kernel of many rows
  int64_t slots = (1 + kWarps) * (all < kMmaRows ? all : kMmaRows);
  if (all > slots) slots = all < kTcRows ? all : kTcRows;
  return ctas * (int64_t)sizeof(int4) + ctas * 2 * slots * (d_kv + 4) * 4;
}

cudaError_t launch_paged_attention(const PagedAttnArgs& g, cudaStream_t st) {
  if (g.n_rows == 0) return cudaSuccess;
  AttnParams a = attn_params(g);
  const int all = a.n_q * a.m, rows = all < kMmaRows ? all : kMmaRows;
  if (paged_attention_tc_fits(g)) {
    const int64_t items = (int64_t)a.S * a.G * ((all + kMmaRows - 1) / kMmaRows);
    if (cluster_size(items, a.cap, g.d_kv == 64 ? Tile<2, 64>::KT : Tile<2, 128>::KT) == 0)
      return launch_paged_attention_tc(g, st);
  }
  a.warp_part = a.part + (int64_t)max_ctas(g.d_kv) * 2 * rows * (g.d_kv + 4);
  if (g.dtype == DT_F32) return g.d_kv == 32 ? run_f32<32>(a, st) : g.d_kv == 64 ? run_f32<64>(a, st) : run_f32<128>(a, st);
  return g.d_kv == 32 ? run_bf16<32>(a, st) : g.d_kv == 64 ? run_bf16<64>(a, st) : run_bf16<128>(a, st);
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
  if (n_rows == 0) return T5_OK;
  PagedAttnArgs a;
  memset(&a, 0, sizeof a);
  rc = paged_pool_args(es, n_kv_heads, d_kv, d_k_pages, d_v_pages, n_pages, page_size, page_stride, slot_stride, head_stride,
                       d_page_table, n_rows / n_q, max_pages, ld_table, &a.pool);
  if (rc != T5_OK) return rc;
  if ((d_bias != nullptr) != (n_bias > 0) || n_bias < 0 || !isfinite(scale)) return T5_ERR_ARG;
  if (!d_q || !d_lens || !d_out || !d_workspace) return T5_ERR_NULL;
  if (ldq < (int64_t)n_heads * d_kv || ldo < (int64_t)n_heads * d_kv) return T5_ERR_ARG;
  if (!paged_aligned(d_q) || !paged_aligned(d_out) || !paged_aligned(d_workspace) || (ldq * es) % 16 || (ldo * es) % 16)
    return T5_ERR_ALIGN;
  if (workspace_bytes < paged_attention_workspace(n_rows, n_q, n_heads, n_kv_heads, d_kv)) return T5_ERR_WORKSPACE;
  a.dtype = dtype; a.n_rows = n_rows; a.n_q = n_q; a.H = n_heads; a.Hkv = n_kv_heads; a.d_kv = d_kv;
  a.q = d_q; a.out = d_out; a.ldq = ldq; a.ldo = ldo; a.lse = d_lse; a.lens = d_lens; a.bias = d_bias; a.n_bias = n_bias;
  a.scale = scale; a.workspace = d_workspace; a.status = g_kernel_status;
  return paged_result(launch_paged_attention(a, (cudaStream_t)stream));
}

}  // extern "C"
