// Attention over a paged cache for many query rows per kv head (several new tokens of heads that share a kv head): the
// products on the tcgen05 tensor cores, bfloat16, heads of 64 and 128 columns.  The formulas, the line of key tiles and its
// shares are those of paged_attention.cu.
//
// With more than 16 rows the kernels there read and multiply every tile once per 16 rows, and their two warps per scheduler
// bound them (64 rows over 4 kv heads of 128 columns, 64 sequences of up to 8192 keys: 343 us for a floor of 82; here 162).
// Here a CTA takes its share of the line in tiles of 64 keys for up to 128 rows at once:
//   S = Q K^T    128 x 64, operands in shared memory, into tensor memory;
//   softmax      thread i owns tensor-memory lane i = one row; its maximum, its sum;
//   O += P V     P as two bfloat16 parts (error 2^-17) in tensor memory, V in shared memory, O in tensor memory.
// An instruction has 128 rows whether they are used or not.  With 64 (32) query rows or fewer the spare lanes hold copies of
// them: copy c takes the c-th half (quarter) of a tile's keys with a maximum and a sum of its own, its weights of the
// other keys are zeros that are written once, and the copies are joined where the item ends.  So every warp has work.
//
// One warp brings keys and values by TMA, as many slots at a time as divide a page (pages of whole multiples of 8 slots; the
// pools are tensors [page][slot][head][column], a key without a page a box outside of them, which reads as zeros), one issues
// the products, four do the softmax, each handing over by mbarriers: S of the next tile is formed beside the softmax of this
// one.  (Two warps with 16-byte asynchronous copies needed 3300 - 4700 cycles for a tile of 32 KB, as much as all the rest.)
// What bounds it: the softmax warps' chain of about 450 instructions a tile, 2700 of the 3300 cycles that a tile of 64 rows
// takes; the products need 930, and the memory brings a tile to each of the two CTAs of an SM in 2800.
#include "paged_attention.cuh"
#include "tc_common.cuh"

namespace {

using namespace tc;

constexpr int kTile = 64;      // keys
constexpr int kMmaWarp = kWarps, kCopyWarp = kWarps + 1, kTcThreads = kThreads + 64;
constexpr int kRing = 4;       // tiles for which it is known which keys exist
constexpr uint32_t kColS = 0, kColP = 64, kColLo = kColP + kTile / 2, kColO = 128, kCols = 256;      // tensor memory

template <int DK, int R> struct TcTile {
  static constexpr int CPR = DK / 8;                       // 16-byte chunks of a row
  static constexpr int Q_BYTES = 128 * DK * 2, KV_BYTES = kTile * DK * 2;
  static constexpr int COPIES = 128 / R, NK = kTile / COPIES;      // keys of a tile that a thread looks at
  static constexpr int K = Q_BYTES, V = K + 2 * KV_BYTES, MISC = V + 2 * KV_BYTES;
  struct Misc {
    uint32_t ok[kRing][2];          // which keys exist
    float2 ml[128];                 // maxima and sums of the copies
    int64_t x0, x1;
    Place place;
    uint64_t go_s, have_p;              // S of the next tile may be written; P is there (a lane of each softmax warp)
    uint64_t have_s, have_o;            // S, O of a tile are there (its products)
    uint64_t full_k[2], full_v[2];      // a stage has landed
    uint64_t free_k[2], free_v[2];      // and has been used (its products)
    uint32_t tmem;
    int abort_flag;
    int plain;                          // the tile's values are taken key by key
  };
  static constexpr int SMEM = MISC + (int)sizeof(Misc) + 1024;
};

template <int N> __device__ __forceinline__ void put_weights(uint32_t at, const uint32_t (&u)[N]) {
  if constexpr (N == 32) tmem_st_32x32b_x32(at, u);
  else if constexpr (N == 16) tmem_st_32x32b_x16(at, u);
  else tmem_st_32x32b_x8(at, u);
}
template <int N> __device__ __forceinline__ void get_scores(uint32_t at, float (&s)[N]) {
  if constexpr (N == 16) {
    uint32_t u[16];
    tmem_ld_32x32b_x16(at, u);
    tmem_wait_ld_dep16(u);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = __uint_as_float(u[i]);
  } else {
    uint32_t u[N / 32][32];
#pragma unroll
    for (int c = 0; c < N / 32; ++c) tmem_ld_32x32b_x32(at + c * 32, u[c]);
#pragma unroll
    for (int c = 0; c < N / 32; ++c) {
      tmem_wait_ld_dep(u[c]);
#pragma unroll
      for (int i = 0; i < 32; ++i) s[c * 32 + i] = __uint_as_float(u[c][i]);
    }
  }
}
// Whether `x` holds in any of the CTA's first kThreads threads; called by those
__device__ __forceinline__ bool any_first(bool x) {
  int y;
  asm volatile("{\n.reg .pred p, q;\nsetp.ne.b32 p, %1, 0;\nbarrier.cta.red.popc.aligned.u32 %0, 1, %2, p;\n}"
               : "=r"(y) : "r"((int)x), "n"(kThreads) : "memory");
  return y != 0;
}
// O += P V of one tile without a product that a row does not see: this lane's weights p of the NK keys of which it sees the
// first n, values from row `key0` of the tile
template <int DK, int NK>
__device__ __noinline__ void values_by_key(const unsigned char* vt, const float* p, int key0, int n, uint32_t o_at, bool first) {
  for (int c = 0; c < DK / 32; ++c) {
    uint32_t o[32];
    if (first) {
#pragma unroll
      for (int i = 0; i < 32; ++i) o[i] = 0;
    } else {
      tmem_ld_32x32b_x32(o_at + c * 32, o);
      tmem_wait_ld_dep(o);
    }
    for (int k = 0; k < NK; ++k) {
      const unsigned char* row = vt + (c >> 1) * (kTile * 128) + (key0 + k) * 128;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint4 u = *reinterpret_cast<const uint4*>(row + ((((c & 1) * 4 + i) ^ ((key0 + k) & 7)) << 4));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if (k < n) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float &x = reinterpret_cast<float&>(o[i * 8 + 2 * e]), &y = reinterpret_cast<float&>(o[i * 8 + 2 * e + 1]);
            x = fmaf(p[k], __uint_as_float(w[e] << 16), x);
            y = fmaf(p[k], __uint_as_float(w[e] & 0xffff0000u), y);
          }
        }
      }
    }
    __syncwarp();
    tmem_st_32x32b_x32(o_at + c * 32, o);
  }
  tmem_wait_st();
}

template <int DK, int R>
__global__ void __launch_bounds__(kTcThreads, 2)
paged_attn_tc_kernel(const __grid_constant__ AttnParams a, const __grid_constant__ CUtensorMap k_map,
                     const __grid_constant__ CUtensorMap v_map, int box_log2) {
  pdl_sync();
  using L = TcTile<DK, R>;
  constexpr int CPR = L::CPR, NK = L::NK, COPIES = L::COPIES;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  typename L::Misc* ms = reinterpret_cast<typename L::Misc*>(smem + L::MISC);
  volatile int* abort_flag = &ms->abort_flag;
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  if (tid == 0) {
    mbar_init(&ms->go_s, kWarps);
    mbar_init(&ms->have_p, kWarps);
    mbar_init(&ms->have_s, 2);
    mbar_init(&ms->have_o, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&ms->full_k[i], 1);
      mbar_init(&ms->full_v[i], 1);
      mbar_init(&ms->free_k[i], 1);
      mbar_init(&ms->free_v[i], 1);
    }
    ms->abort_flag = 0;
    fence_barrier_init();
  }
  if (w == kMmaWarp) tmem_alloc(&ms->tmem, kCols);
  if (tid < kThreads) {
    int64_t x0, x1;
    Place p = {};
    find_share(a, kTile, x0, x1, p);
    if (tid == 0) { ms->x0 = x0; ms->place = p; }      // the CTA's share is that of its first kWarps warps
    if (tid == kThreads - 32) ms->x1 = x1;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  Place cur = ms->place;
  const int n = (int)(ms->x1 - ms->x0);
  const uint32_t tmem = ms->tmem, smem_s = smem_u32(smem);
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    const bool ok = mbar_wait(bar, parity, abort_flag, a.status, PAGED_TIMEOUT);
    return (bool)__all_sync(0xffffffffu, ok);
  };

  if (w == kCopyWarp) {
    // ------------------------------------------------------------ keys and values: lane i looks up box i of a tile
    const int boxes = kTile >> box_log2, box = 1 << box_log2;
    const uint32_t lead = elect_one_lane();
    auto look = [&]() { return lane < boxes ? page_entry(a, cur, cur.blk * kTile + lane * box) : kNoKey; };
    struct Boxes { int page[kTile / 8], slot[kTile / 8], head; };      // of a tile
    auto load = [&](const CUtensorMap* map, const Boxes& x, int to, uint64_t* full) {
      if (lead) {      // one lane for all boxes: lanes of a warp would only take turns
        mbar_arrive_expect_tx(full, L::KV_BYTES);
#pragma unroll
        for (int i = 0; i < kTile / 8; ++i) {
          if (i == boxes) break;
#pragma unroll
          for (int c = 0; c < DK / 64; ++c)
            tma_load_4d(smem + to + c * (kTile * 128) + i * box * 128, map, c * 64, x.head, x.slot[i], x.page[i], full);
        }
      }
      __syncwarp();
    };
    int entry = n > 0 ? look() : kNoKey, out_k = 0, out_v = 0;      // out_*: tiles sent for
    Boxes now = {}, last;
    // Keys go a tile ahead of the values, as scores do of outputs: sent for together, the keys of a tile waited for the
    // output of the one three before it (24 rows, 64 sequences of up to 8192 keys: 126 instead of 120 us)
    for (int t = 0; t <= n && n > 0; ++t) {
      last = now;
      if (t < n) {
        const int first_key = cur.blk * kTile, key = first_key + lane * box, keys = cur.len - first_key;
        const int slot = lane < boxes ? key - (int)a.pool.ps.div(key) * a.pool.page_size : 0;
        const int page = page_of(a, entry), at = page < 0 ? a.pool.n_pages : page;
        const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
        const uint32_t low = __ballot_sync(0xffffffffu, ((there >> (lane >> box_log2)) & 1) && lane < keys);
        const uint32_t high = __ballot_sync(0xffffffffu, ((there >> ((lane + 32) >> box_log2)) & 1) && lane + 32 < keys);
        now.head = (int)a.by_tiles.div(cur.k);
        step(a, kTile, cur);
        if (t + 1 < n) entry = look();
#pragma unroll
        for (int i = 0; i < kTile / 8; ++i) {
          now.page[i] = __shfl_sync(0xffffffffu, at, i);
          now.slot[i] = __shfl_sync(0xffffffffu, slot, i);
        }
        if (t >= 2 && !wait(&ms->free_k[t & 1], ((t >> 1) - 1) & 1)) break;
        if (lead) { ms->ok[t % kRing][0] = low; ms->ok[t % kRing][1] = high; }
        load(&k_map, now, L::K + (t & 1) * L::KV_BYTES, &ms->full_k[t & 1]);
        out_k = t + 1;
      }
      if (t >= 1) {
        const int v = t - 1;
        if (v >= 2 && !wait(&ms->free_v[v & 1], ((v >> 1) - 1) & 1)) break;
        load(&v_map, last, L::V + (v & 1) * L::KV_BYTES, &ms->full_v[v & 1]);
        out_v = t;
      }
    }
    // no copy may be on its way when the CTA ends (with a limit, should a wait above have given up)
    const long long t0 = clock64();
    auto landed = [&](uint64_t* full, int tile) {
      while (!mbar_try_wait(&full[tile & 1], (tile >> 1) & 1) && clock64() - t0 < kWaitCycles) {}
    };
    for (int i = 1; i <= 2; ++i) {
      if (out_k >= i) landed(ms->full_k, out_k - i);
      if (out_v >= i) landed(ms->full_v, out_v - i);
    }
  } else if (w == kMmaWarp) {
    // ------------------------------------------------------------ products
    const uint32_t lQ = desc_lo_k(smem_s), lK = desc_lo_k(smem_s + L::K), lV = desc_lo_mn(smem_s + L::V);
    constexpr uint32_t idesc_s = make_idesc(128, kTile, false, false), idesc_o = make_idesc(128, DK, false, true);
    const uint32_t lead = elect_one_lane();
    auto scores = [&](int t) {
      if (!wait(&ms->full_k[t & 1], (t >> 1) & 1) || !wait(&ms->go_s, t & 1)) return false;
      tc_fence_after();
      const uint32_t k = lK + (((t & 1) * L::KV_BYTES) >> 4);
#pragma unroll
      for (int kk = 0; kk < DK / 16; ++kk)
        umma_bf16_lo_lead(tmem + kColS, lQ + (((kk >> 2) * 16384 + (kk & 3) * 32) >> 4),
                          k + (((kk >> 2) * (kTile * 128) + (kk & 3) * 32) >> 4), idesc_s, kk != 0, lead);
      umma_commit_lead(&ms->have_s, lead);
      if (lead) mbar_arrive(&ms->have_s);      // passes on which keys exist
      umma_commit_lead(&ms->free_k[t & 1], lead);
      return true;
    };
    bool ok = n == 0 || scores(0), first = true;
    for (int u = 0; u < n && ok; ++u) {
      const bool piece_ends = cur.blk + 1 == cur.nb || u + 1 == n;
      if (!piece_ends) ok = scores(u + 1);      // beside the softmax of this tile; an item's first S waits for its Q
      if (!ok || !wait(&ms->full_v[u & 1], (u >> 1) & 1) || !wait(&ms->have_p, u & 1)) break;
      tc_fence_after();
      if (ms->plain == 0) {
        const uint32_t v = lV + (((u & 1) * L::KV_BYTES) >> 4);
#pragma unroll
        for (int ks = 0; ks < kTile / 16; ++ks) {
          umma_bf16_ta_lead(tmem + kColO, tmem + kColP + ks * 8, v + ((ks * 2048) >> 4), idesc_o, !first || ks != 0, lead);
          umma_bf16_ta_lead(tmem + kColO, tmem + kColLo + ks * 8, v + ((ks * 2048) >> 4), idesc_o, 1, lead);
        }
      }
      umma_commit_lead(&ms->have_o, lead);
      umma_commit_lead(&ms->free_v[u & 1], lead);
      first = piece_ends;
      step(a, kTile, cur);
      if (piece_ends && u + 1 < n) ok = scores(u + 1);
    }
  } else {
    // ------------------------------------------------------------ softmax: thread = lane of tensor memory = row
    const uint32_t mine = tmem + ((uint32_t)(w * 32) << 16);
    const int r = tid % R, part = tid / R;      // row of the tile, copy
    if (COPIES > 1) {
      uint32_t none[32] = {};
      tmem_st_32x32b_x32(mine + kColP, none);
      tmem_st_32x32b_x32(mine + kColLo, none);
      tmem_wait_st();
    }
    auto arrive = [&](uint64_t* bar) {
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
    };
    int row = 0, h = 0;
    int len = 0, min_len = 0, all_len = 0;      // keys this row sees; the fewest that a row of the warp, of the sequence sees
    bool valid = false, fresh = true, first = true, ok = true;
    const float* bias = a.bias;
    float m = -INFINITY, l = 0.f, far = 0.f;
    uint32_t phase_o = 0;
    Pieces pieces;
    pieces.starts_here = cur.blk == 0;
    for (int u = 0; u < n && ok; ++u) {
      const bool item_ends = cur.blk + 1 == cur.nb, piece_ends = item_ends || u + 1 == n;
      if (fresh) {      // the item's query rows, once per copy
        const Rows rows(a, cur, R);
#pragma unroll
        for (int i = 0; i < (R * CPR + kThreads - 1) / kThreads; ++i) {
          const int idx = i * kThreads + tid, qr = idx / CPR, c = idx % CPR;
          uint4 q = make_uint4(0, 0, 0, 0);
          if (qr < rows.n) {
            int q_row, q_h;
            rows.place(a, cur, qr, q_row, q_h);
            q = *reinterpret_cast<const uint4*>(a.q + (int64_t)q_row * a.ldq + q_h * (DK * 2) + c * 16);
          }
#pragma unroll
          for (int k = 0; k < COPIES; ++k) {
            const int at = k * R + qr;
            *reinterpret_cast<uint4*>(smem + (c / 8) * 16384 + at * 128 + (((c % 8) ^ (at & 7)) << 4)) = q;
          }
        }
        fence_proxy_async();
        tc_fence_before();
        arrive(&ms->go_s);
        valid = r < rows.n;
        rows.place(a, cur, valid ? r : 0, row, h);
        len = valid ? (a.n_q == 1 ? cur.len : row_len(a, row)) : 0;
        min_len = valid ? len : 0x7fffffff;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) min_len = min(min_len, __shfl_xor_sync(0xffffffffu, min_len, o));
        all_len = cur.len;
        for (int i = 0; a.n_q > 1 && i < a.n_q; ++i) all_len = min(all_len, row_len(a, cur.s * a.n_q + i));
        if (a.bias != nullptr) { bias = a.bias + (int64_t)h * a.n_bias; far = bias[0]; }
        m = -INFINITY; l = 0.f; first = true; fresh = false;
      }
      ok = wait(&ms->have_s, u & 1);
      if (!ok) break;
      tc_fence_after();
      const int k0 = cur.blk * kTile + part * NK;      // the first of this lane's keys
      float s[NK];
      get_scores<NK>(mine + kColS + part * NK, s);
      if (!piece_ends) {
        tc_fence_before();
        arrive(&ms->go_s);
      }
      if (a.bias != nullptr && a.n_bias - min_len + k0 + NK - 1 > 0) {
        const int at = a.n_bias - len + k0;
#pragma unroll
        for (int i = 0; i < NK; ++i) s[i] = fmaf(s[i], a.scale, bias[min(max(at + i, 0), a.n_bias - 1)]);
      } else {
#pragma unroll
        for (int i = 0; i < NK; ++i) s[i] = fmaf(s[i], a.scale, far);
      }
      const uint32_t ok0 = ms->ok[u % kRing][0], ok1 = ms->ok[u % kRing][1];
      if ((ok0 & ok1) != 0xffffffffu || k0 + NK > min_len) {
        const uint64_t have = (((uint64_t)ok1 << 32) | ok0) >> (part * NK);
#pragma unroll
        for (int i = 0; i < NK; ++i)
          if (!((have >> i) & 1) || k0 + i >= len) s[i] = -INFINITY;
      }
      float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int i = 0; i < NK; ++i) top[i & 3] = fmaxf(top[i & 3], s[i]);
      const float m_tile = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
      // The reference point of a row follows its maximum when that has grown by more than 5 (weights up to e^5 are as good
      // as weights up to 1), so that O is rescaled in tensor memory only then
      const bool grow = m_tile > m + 5.f || (m == -INFINITY && m_tile != -INFINITY);
      const bool moves = __any_sync(0xffffffffu, grow);
      const float m_new = moves ? fmaxf(m, m_tile) : m, ref = m_new == -INFINITY ? 0.f : m_new;
      const float corr = ex2((m - ref) * kLog2e);
      float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < NK; ++i) {
        s[i] = ex2((s[i] - ref) * kLog2e);      // differences first: a bias of the lowest float stays finite
        sum[i & 3] += s[i];
      }
      l = (moves ? l * corr : l) + ((sum[0] + sum[1]) + (sum[2] + sum[3]));
      m = m_new;
      if (!first) {      // the products with the last tile's weights are done: O and the weights may change
        ok = wait(&ms->have_o, phase_o);
        phase_o ^= 1;
        if (!ok) break;
        tc_fence_after();
        if (moves) {
#pragma unroll
          for (int c = 0; c < DK / 32; ++c) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(mine + kColO + c * 32, o);
            tmem_wait_ld_dep(o);
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * corr);
            tmem_st_32x32b_x32(mine + kColO + c * 32, o);
          }
        }
      }
      constexpr int W = NK / 2 < 16 ? NK / 2 : 16;      // columns of weights at a time
#pragma unroll
      for (int b = 0; b < NK / 2; b += W) {
        uint32_t hi[W], lo[W];
#pragma unroll
        for (int i = 0; i < W; ++i) split2(s[2 * (b + i)], s[2 * (b + i) + 1], hi[i], lo[i]);
        put_weights(mine + kColP + part * (NK / 2) + b, hi);
        put_weights(mine + kColLo + part * (NK / 2) + b, lo);
      }
      tmem_wait_st();
      bool plain = false;
      unsigned char* vt = smem + L::V + (u & 1) * L::KV_BYTES;
      const int keys = cur.len - cur.blk * kTile;      // of this tile and behind it
      if (keys < kTile || all_len < (cur.blk + 1) * kTile) {
        ok = wait(&ms->full_v[u & 1], (u >> 1) & 1);
        if (!ok) break;
      }
      // Slots behind the last key may hold anything and have weight 0: 0 x NaN would spoil the row, so they become zeros.
      if (keys < kTile) {
        for (int i = max(keys, 0) * CPR + tid; i < kTile * CPR; i += kThreads)
          *reinterpret_cast<uint4*>(vt + (i % CPR / 8) * (kTile * 128) + i / CPR * 128 + (i % 8) * 16) = make_uint4(0, 0, 0, 0);
        fence_proxy_async();
        sync_first();
      }
      // Keys that one row sees and another does not have weight 0 there as well: if such a tile holds a value that is not
      // finite, it is taken key by key.
      if (all_len < min((cur.blk + 1) * kTile, cur.len)) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < L::KV_BYTES / 16 / kThreads; ++i) {
          const uint4 v = *reinterpret_cast<const uint4*>(vt + (i * kThreads + tid) * 16);
          bad |= not_finite(v.x) | not_finite(v.y) | not_finite(v.z) | not_finite(v.w);
        }
        plain = any_first(bad);
        if (plain) {
          float p[NK];      // a copy, so that the rare call does not push the registers of the others into memory
#pragma unroll
          for (int i = 0; i < NK; ++i) p[i] = s[i];
          values_by_key<DK, NK>(vt, p, part * NK, len - k0, mine + kColO, first);
        }
      }
      if (tid == 0) ms->plain = plain;
      tc_fence_before();
      arrive(&ms->have_p);
      first = false;
      if (piece_ends) {
        ok = wait(&ms->have_o, phase_o);
        phase_o ^= 1;
        if (!ok) break;
        tc_fence_after();
        float mx = m, lt = l, e = 1.f;      // of all copies; this one's share
        if (COPIES > 1) {
          ms->ml[tid] = make_float2(m, l);
          sync_first();
#pragma unroll
          for (int k = 0; k < COPIES; ++k) mx = fmaxf(mx, ms->ml[k * R + r].x);
          const float to_ref = mx == -INFINITY ? 0.f : mx;
          lt = 0.f;
#pragma unroll
          for (int k = 0; k < COPIES; ++k) lt += ex2((ms->ml[k * R + r].x - to_ref) * kLog2e) * ms->ml[k * R + r].y;
          e = ex2((m - to_ref) * kLog2e);
        }
        const bool whole = pieces.whole(item_ends);
        const float f = !whole ? e : (lt == 0.f ? 0.f : e / lt);
        bf16* out = out_row<bf16, DK>(a, row, h);
        float* pt = a.part + (((int64_t)blockIdx.x * 2 + pieces.slot()) * a.rows + r) * kRowOf<DK>;
        float* join = reinterpret_cast<float*>(smem);      // over the query rows: [32 columns][copies but the first][R]
#pragma unroll 1
        for (int c = 0; c < DK / 32; ++c) {
          uint32_t u32[32];
          float o[32];
          __syncwarp();
          tmem_ld_32x32b_x32(mine + kColO + c * 32, u32);
          tmem_wait_ld_dep(u32);
#pragma unroll
          for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(u32[i]) * f;
          if (COPIES > 1) {
            if (part > 0) {
#pragma unroll
              for (int i = 0; i < 32; ++i) join[i * (128 - R) + tid - R] = o[i];
            }
            sync_first();
            if (part == 0) {
#pragma unroll
              for (int i = 0; i < 32; ++i)
#pragma unroll
                for (int k = 1; k < COPIES; ++k) o[i] += join[i * (128 - R) + (k - 1) * R + r];
            }
            sync_first();
          }
          if (part == 0 && valid) {
            if (whole) {
#pragma unroll
              for (int i = 0; i < 32; i += 8) {
                uint32_t b[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                  const __nv_bfloat162 two = __floats2bfloat162_rn(o[i + 2 * k], o[i + 2 * k + 1]);
                  b[k] = *reinterpret_cast<const uint32_t*>(&two);
                }
                *reinterpret_cast<uint4*>(out + c * 32 + i) = make_uint4(b[0], b[1], b[2], b[3]);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 32; i += 4)
                *reinterpret_cast<float4*>(pt + c * 32 + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
            }
          }
        }
        if (part == 0 && valid) {
          if (whole) write_lse(a, row, h, mx, lt);
          else { pt[DK] = mx; pt[DK + 1] = lt; }
        }
        pieces.note(a, cur, item_ends);
        fresh = true;
        sync_first();      // maxima and sums have been read
      }
      step(a, kTile, cur);
    }
    if (tid == 0) a.meta[blockIdx.x] = pieces.meta;
  }
  tc_fence_before();
  __syncthreads();
  if (w == kMmaWarp) {
    tc_fence_after();
    tmem_dealloc(tmem, kCols);
  }
}

// The pool as a tensor [page][slot][head][column], read in boxes of 64 columns of `box` slots
bool pool_map(CUtensorMap* map, void* base, const PagedAttnArgs& g, int box) {
  const EncodeTiledFn encode = get_encode();
  if (encode == nullptr) return false;
  const cuuint64_t size[4] = {(cuuint64_t)g.d_kv, (cuuint64_t)g.Hkv, (cuuint64_t)g.pool.page_size, (cuuint64_t)g.pool.n_pages};
  const cuuint64_t stride[3] = {(cuuint64_t)g.pool.head_stride, (cuuint64_t)g.pool.slot_stride, (cuuint64_t)g.pool.page_stride};
  const cuuint32_t part[4] = {64, 1, (cuuint32_t)box, 1}, one[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, base, size, stride, part, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DK, int R>
cudaError_t run(AttnParams& a, const CUtensorMap& k_map, const CUtensorMap& v_map, int box_log2, cudaStream_t st) {
  constexpr int smem = TcTile<DK, R>::SMEM;
  static_assert(2 * (smem + 1024 + 256) <= 228 * 1024, "two CTAs per SM");
  static std::atomic<int> known[64];      // SMs, by device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  int sms = known[dev].load(std::memory_order_acquire);
  if (sms == 0) {
    e = cudaFuncSetAttribute(paged_attn_tc_kernel<DK, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    known[dev].store(sms, std::memory_order_release);
  }
  set_tiles(a, R);
  const int ctas = 2 * sms < max_ctas(DK) ? 2 * sms : max_ctas(DK);
  a.by_workers = FastDiv(ctas * kWarps);
  a.extra = a.bias != nullptr ? 2 : 1;
  e = launch_pdl(paged_attn_tc_kernel<DK, R>, dim3(ctas), dim3(kTcThreads), (size_t)smem, st, a, k_map, v_map, box_log2);
  if (e != cudaSuccess) return e;
  return launch_join<bf16, DK, R>(a, ctas, st);
}
template <int DK>
cudaError_t run_rows(AttnParams& a, const CUtensorMap& k, const CUtensorMap& v, int box_log2, cudaStream_t st) {
  const int rows = a.n_q * a.m;
  if (rows <= 32) return run<DK, 32>(a, k, v, box_log2, st);
  return rows <= 64 ? run<DK, 64>(a, k, v, box_log2, st) : run<DK, 128>(a, k, v, box_log2, st);
}

}  // namespace

// More rows than one tile of the kernels for few, and, for two tiles of those, caches that may be long: an item costs more
// here and a tile less.  Measured, us there / here, 32 rows over 8 kv heads of 128 columns: 128 sequences of up to 300 keys
// 59 / 72, 32 of up to 1000 44 / 40; 4 kv heads, 64 sequences of up to 8192 183 / 120; 40 rows, up to 300 keys 53 / 50, up to
// 8192 261 / 148.
bool paged_attention_tc_fits(const PagedAttnArgs& g) {
  const int64_t limit = 1ll << 40;      // of a tensor's strides
  const int rows = g.n_q * (g.H / g.Hkv);
  return g.dtype == DT_BF16 && g.d_kv >= 64 && g.pool.page_size % 8 == 0 &&
         (rows > 2 * kMmaRows || (rows > kMmaRows && g.pool.max_pages * g.pool.page_size > 512)) &&
         g.pool.page_stride < limit && g.pool.slot_stride < limit && g.pool.head_stride < limit;
}

cudaError_t launch_paged_attention_tc(const PagedAttnArgs& g, cudaStream_t st) {
  AttnParams a = attn_params(g);
  CUtensorMap k, v;
  int box_log2 = 3;      // boxes of 8 slots, or as many more as a page is a multiple of
  while ((1 << box_log2) < kTile && g.pool.page_size % (2 << box_log2) == 0) ++box_log2;
  if (!pool_map(&k, g.pool.k, g, 1 << box_log2) || !pool_map(&v, g.pool.v, g, 1 << box_log2)) return cudaErrorInvalidValue;
  return g.d_kv == 64 ? run_rows<64>(a, k, v, box_log2, st) : run_rows<128>(a, k, v, box_log2, st);
}
