// Paged attention of drafted-token trees (mcpu_tree_attention_forward) on the
// 5th-generation tensor cores (tcgen05 + TMEM).
//
// o_t = sum_{j in V(t)} e^{s_j - m} v_j / sum_{j in V(t)} e^{s_j - m},  s_j = scale q_t . k_j
// where V(t) holds the row's context keys (inside the window of t's position)
// and the nodes whose bit is set in t's mask.
//
// Work: an item is one (row, kv head, tile of 256 query rows = 256 / g nodes x
// the g heads); it walks the row's keys in blocks of 128 (8 pages). The blocks
// of all items, weighted by what a block costs, form one line that is cut into
// equal pieces, one per CTA (one CTA per SM): whatever the lengths, every SM
// gets the same share, and an item that crosses a cut is computed in parts
// that merge_tree_kernel joins by log-sum-exp in the order of the CTAs. Every
// CTA derives the line from seq_lens and query_start_loc itself (a prefix sum
// over the rows), so there is no planning launch.
//
// One CTA, 12 warps:
//   warps 0-3  softmax of tile A, warps 4-7 of tile B: thread t owns row
//              t & 127 (TMEM lane). Running max and sum in fp32, P to TMEM as
//              bf16 (as the append kernel does, the rounding of each p_j is
//              2^-8 relative at most), O rescaled only when the max rises by
//              more than 2^8;
//   warps 8, 11  producers: find the CTA's parts, load query tiles and K (8) and V
//              (11) blocks by TMA into a ring each;
//   warps 9, 10  MMA issuers of tile A and B: S = Q K^T (M 128, N 128, K 64),
//              then O += P V (M 128, N 64, K 128, P from TMEM).
// An item with more than 128 query rows runs as two tiles over the same K/V
// blocks. One with at most 128 rows (up to 16 nodes at g = 8) would leave
// tile B idle, so the two tiles then hold the same rows and take alternate key
// blocks; their two states are joined in shared memory at the end.
//
// Waits are bounded (common.cuh); one that runs out raises an abort flag that
// ends every role, and TMEM is freed after the issuers' MMAs have drained.
#include "tcgen05.cuh"
#include "tree_round.cuh"

namespace mcpu {

namespace {

constexpr int kTileRows = 128;  // query rows of one tile (TMEM lanes)
constexpr int kItemRows = 256;
constexpr int kBlockKeys = 128;
constexpr int kBlockPages = kBlockKeys / kPage;
constexpr int kBlockBytes = kBlockKeys * kRowBytes;  // one K or V block: 16 KiB
constexpr int kKStages = 4, kVStages = 4;
constexpr int kQBytes = kItemRows * kRowBytes;
constexpr int kTileQBytes = kTileRows * kRowBytes;
constexpr int kProducerWarpK = 8, kIssueWarpA = 9, kProducerWarpV = 11;
constexpr int kTreeThreads = 384;
constexpr uint32_t kTmemCols = 512;
// cost of a part's set-up and end, of a block walked by both tiles, and of a
// block that one of two alternating tiles walks
constexpr int kCostItem = 2, kCostPair = 2, kCostAlt = 1;
constexpr int kMinQuota = 4;  // smallest piece of the line worth a CTA of its own
constexpr float kRescale = 8.f;  // log2 units: P may reach 2^8 before O is rescaled
constexpr int kStateRows = kHeadDim + 2;  // O, m and l of a row in the exchange buffer
constexpr int kXchBytes = kStateRows * kTileRows * 4;

// TMEM columns of tile x
__device__ __forceinline__ uint32_t col_s(int x) { return x ? 128u : 0u; }
__device__ __forceinline__ uint32_t col_o(int x) { return x ? 320u : 256u; }
__device__ __forceinline__ uint32_t col_p(int x) { return x ? 448u : 384u; }

struct Part {  // a run of key blocks of one item
  int32_t row;  // -1: no more parts
  int32_t token, n_tok, node;  // first query token, tokens, first node of the tile
  int32_t ctx, len, kvh;
  int32_t kb0, key_begin;  // key of block 0 (a page start), first key any node can see
  int32_t b0, b1;
  int32_t slot;  // partial slot, or -1: the part is the whole item
  int32_t alt;
};

struct TreeSmem {
  uint64_t q_full, q_empty;
  uint64_t k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
  uint64_t s_full[2], s_free[2], p_full[2], o_ready[2], o_free[2];
  uint64_t part_full[2], part_empty[2];
  uint64_t xch_full, xch_empty;
  uint64_t drain[2];
  Part parts[2];
  int64_t scan[kTreeThreads / 32];
  uint32_t tmem_base;
  int32_t abort_flag;
};

size_t tree_smem_bytes() {
  return 1024 + kQBytes + (size_t)(kKStages + kVStages) * kBlockBytes + kXchBytes + sizeof(TreeSmem) +
         sizeof(int64_t) * (kMaxSeqs + 1);
}

// ------------------------------------------------------------ the work line
struct RowGeom {
  int q0, L, S, C, key_begin, kb0, nb, tiles;
  int64_t pair_cost, last_cost;  // of the row's full tiles and of its last one
  __device__ int64_t head_cost() const { return (tiles - 1) * pair_cost + last_cost; }
};

// Geometry of row r; false (L = 0: nothing wrong) if it has no work, with the
// status bits of what is wrong.
__device__ __forceinline__ bool row_geom(const TreeParams& p, int r, RowGeom* w, int32_t* bits) {
  w->q0 = __ldg(p.qsl + r);
  w->L = __ldg(p.qsl + r + 1) - w->q0;
  w->S = __ldg(p.seq_lens + r);
  if (w->L == 0) return false;
  if (w->q0 < 0 || w->L < 0 || w->L > p.total_q - w->q0 || w->S < w->L || w->S > p.max_pages * kPage) {
    *bits |= kStatusBadLengths;
    return false;
  }
  if (w->L > 32 * p.words) {
    *bits |= kStatusUnsupportedRow;
    return false;
  }
  w->C = w->S - w->L;
  // positions count as at least C, so no node sees a key before C - W + 1
  w->key_begin = p.window > 0 ? max(0, w->C - p.window + 1) : 0;
  w->kb0 = w->key_begin / kPage * kPage;
  w->nb = (w->S - w->kb0 + kBlockKeys - 1) / kBlockKeys;
  const int rows = w->L * p.group;
  w->tiles = (rows + kItemRows - 1) / kItemRows;
  const int last = rows - (w->tiles - 1) * kItemRows;
  w->pair_cost = kCostItem + (int64_t)w->nb * kCostPair;
  w->last_cost = last <= kTileRows ? kCostItem + (int64_t)w->nb * kCostAlt : w->pair_cost;
  return true;
}

// Blocks of an item of `nb` blocks that lie before `x` units of it.
__device__ __forceinline__ int blocks_before(int64_t x, int nb, int64_t cost) {
  if (x <= kCostItem) return 0;
  if (x >= cost) return nb;
  // cost = kCostItem + nb * weight, weight 1 or 2
  const int64_t weight = cost - kCostItem == nb ? 1 : kCostPair;
  const int64_t b = (x - kCostItem + weight - 1) / weight;
  return b < nb ? (int)b : nb;
}

// ------------------------------------------------------------------- waits
__device__ __forceinline__ bool wait_sleep(uint32_t bar, uint32_t parity, volatile int32_t* abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait_sleep(bar, parity, 10000)) {
    if (*abort_flag) return false;
    if (global_timer_ns() - t0 > kWaitTimeoutNs) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}
__device__ __forceinline__ bool wait_poll(uint32_t bar, uint32_t parity, volatile int32_t* abort_flag) {
  if (mbar_try_wait(bar, parity)) return true;
  const uint64_t t0 = global_timer_ns();
  while (!mbar_try_wait(bar, parity)) {
    if (*abort_flag) return false;
    if (global_timer_ns() - t0 > kWaitTimeoutNs) {
      *abort_flag = 1;
      return false;
    }
  }
  return true;
}

// A 2-D box load issued by one elected lane of a warp that runs in step: its
// operands stay in the uniform datapath (from a lone lane every operand is
// moved there first, which made the issue of a block's 16 boxes take longer
// than their transfer).
__device__ __forceinline__ void tma_load_2d_e(uint32_t dst, const CUtensorMap* map, int32_t y, uint32_t bar,
                                              uint64_t policy) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint"
      " [%0], [%1, {%2, %3}], [%4], %5;\n\t}" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(0), "r"(y), "r"(bar), "l"(policy)
      : "memory");
}
__device__ __forceinline__ void arrive_expect_tx_e(uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t.reg .pred e;\n\telect.sync _|e, 0xffffffff;\n\t"
      "@e mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t}" ::"r"(bar),
      "r"(bytes)
      : "memory");
}

// ------------------------------------------------------------------ softmax
// the low n bits (none for n <= 0, all for n >= 32)
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

__device__ __forceinline__ void hide(uint32_t (&sv)[32], uint32_t seen) {
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!(seen >> e & 1u)) sv[e] = 0xff800000u;
}

__device__ __forceinline__ float scores_max(const uint32_t (&sv)[2][32]) {
  float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int e = 0; e < 32; e += 8)
#pragma unroll
      for (int k = 0; k < 4; ++k)
        m[k] = fmax3(m[k], __uint_as_float(sv[c][e + 2 * k]), __uint_as_float(sv[c][e + 2 * k + 1]));
  return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}

// pk = bf16(2^(s * scale - mu)); returns their fp32 sum (before rounding)
__device__ __forceinline__ float weights(const uint32_t (&sv)[2][32], float scale_log2, float neg_mu,
                                         uint32_t (&pk)[32]) {
  const uint64_t sc = pack_f32x2(scale_log2, scale_log2), mu = pack_f32x2(neg_mu, neg_mu);
  uint64_t sum[2] = {0, 0};
#pragma unroll
  for (int c = 0; c < 2; ++c)
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      const uint64_t x = fma2((uint64_t)sv[c][e] | ((uint64_t)sv[c][e + 1] << 32), sc, mu);
      const float p0 = ex2_approx(lo_f32(x)), p1 = ex2_approx(hi_f32(x));
      sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pack_f32x2(p0, p1));
      pk[c * 16 + e / 2] = pack_bf16x2(p0, p1);
    }
  const uint64_t s = add2(sum[0], sum[1]);
  return lo_f32(s) + hi_f32(s);
}

// Weights of 64 scores against the reference m_ref (log2 units). A sum below
// 2^8 shows that no weight exceeds 2^8, so the maximum is only taken when it
// does not (or before the first reference): then m_ref rises if the maximum
// exceeds it by more than kRescale, and alpha takes the factor for earlier
// weights.
__device__ __forceinline__ float chunk_weights(const uint32_t (&sv)[2][32], float scale_log2, float& m_ref,
                                               float& alpha, uint32_t (&pk)[32]) {
  float sum = 0.f;
  bool redo = m_ref == -INFINITY;
  if (!redo) {
    sum = weights(sv, scale_log2, -m_ref, pk);
    redo = !(sum < 256.f);
  }
  if (redo) {
    const float mx = scores_max(sv) * scale_log2;
    if (mx > m_ref + kRescale) {
      alpha *= ex2_approx(m_ref - mx);  // 0 before the first reference
      m_ref = mx;
    }
    sum = weights(sv, scale_log2, m_ref == -INFINITY ? 0.f : -m_ref, pk);
  }
  return sum;
}

__device__ __forceinline__ void zero_smem16(uint32_t addr) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0u) : "memory");
}

// What the masks say about the block of keys at kb: seen[c], the keys kb + 32c ..
// that the thread's node (token t, window from key lo) sees; returns whether
// the slot kb + 32 wq + lane holds a V row that no node of the row sees.
__device__ __forceinline__ bool block_masks(const TreeParams& p, const Part& a, int t, int lo, int kb, int wq, int lane,
                                            uint32_t (&seen)[4]) {
  const int ctx = a.ctx, len = a.len, j = kb + 32 * wq + lane;
  uint32_t mw[5] = {0, 0, 0, 0, 0};
  const int n0 = kb - ctx, w0 = n0 >> 5;  // node of the block's first key, and its mask word
  bool dead = j < a.key_begin;
  if (n0 > -kBlockKeys) {
#pragma unroll
    for (int c = 0; c < 5; ++c)
      if (w0 + c >= 0 && w0 + c < p.words) mw[c] = __ldg(p.mask + (size_t)t * p.words + w0 + c);
    uint32_t u0 = 0, u1 = 0;  // union over the row's nodes of the two words with this warp's slots
    for (int k = lane; k < len - ctx; k += 32) {
      const uint32_t* m = p.mask + (size_t)(a.token - a.node + k) * p.words;
      if (w0 + wq >= 0 && w0 + wq < p.words) u0 |= __ldg(m + w0 + wq);
      if (w0 + wq + 1 >= 0 && w0 + wq + 1 < p.words) u1 |= __ldg(m + w0 + wq + 1);
    }
    u0 = __reduce_or_sync(0xffffffffu, u0);
    u1 = __reduce_or_sync(0xffffffffu, u1);
    const uint32_t any = __funnelshift_r(u0, u1, n0 & 31);
    // past the row's end only its last page holds anything: later pages arrive as zeros
    dead |= j >= len ? j < ((len + kPage - 1) & ~(kPage - 1)) : j >= ctx && !(any >> lane & 1u);
  }
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int k0 = kb + 32 * c;
    seen[c] = (low_bits(ctx - k0) & ~low_bits(lo - k0)) |
              (__funnelshift_r(mw[c], mw[c + 1], n0 & 31) & low_bits(len - k0));
  }
  return dead;
}

__device__ __forceinline__ float tree_sink(const TreeParams& p, int h) {
  return p.sinks ? p.sinks[h] * 1.4426950408889634f : -INFINITY;
}

// --------------------------------------------------------------- the kernel
__global__ void __launch_bounds__(kTreeThreads, 1)
    tree_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap qmap_alt,
                const TreeParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  const uint32_t sQ = base, sK = sQ + kQBytes, sV = sK + kKStages * kBlockBytes;
  uint8_t* after = smem_raw + (base - raw) + kQBytes + (kKStages + kVStages) * kBlockBytes;
  float* xch = reinterpret_cast<float*>(after);  // [kStateRows][kTileRows]
  TreeSmem& st = *reinterpret_cast<TreeSmem*>(after + kXchBytes);
  int64_t* prefix = reinterpret_cast<int64_t*>(after + kXchBytes + sizeof(TreeSmem));
  volatile int32_t* abort_flag = &st.abort_flag;
  auto bar = [&](uint64_t& b) { return smem_addr(&b); };
  const int B = p.num_seqs, g = p.group, Hkv = p.num_kv_heads, Hq = p.num_q_heads;

  if (p.qsl[0] != 0 || p.qsl[B] != p.total_q) {
    if (blockIdx.x == 0 && threadIdx.x == 0) {
      atomicOr(p.status, kStatusBadLengths);
      p.plan[0] = 0;
    }
    return;
  }
  // ---- the work line: prefix[r] = cost of the rows before r
  {
    const int per = (B + kTreeThreads - 1) / kTreeThreads;
    const int r0 = min(B, (int)threadIdx.x * per), r1 = min(B, r0 + per);
    int64_t mine = 0;
    int32_t bits = 0;
    RowGeom w;
    for (int r = r0; r < r1; ++r)
      if (row_geom(p, r, &w, &bits)) mine += w.head_cost() * Hkv;
    if (bits && blockIdx.x == 0) atomicOr(p.status, bits);
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, (long long)incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) st.scan[warp] = incl;
    __syncthreads();
    int64_t at = incl - mine;
    for (int i = 0; i < warp; ++i) at += st.scan[i];
    for (int r = r0; r < r1; ++r) {
      prefix[r] = at;
      if (row_geom(p, r, &w, &bits)) at += w.head_cost() * Hkv;
    }
    if ((int)threadIdx.x == kTreeThreads - 1) {
      prefix[B] = at;
      if (B == 0) prefix[0] = 0;
    }
  }
  if (threadIdx.x == 0) {
    mbar_init(bar(st.q_full), 1);
    mbar_init(bar(st.q_empty), 2);
    for (int s = 0; s < kKStages; ++s) {
      mbar_init(bar(st.k_full[s]), 1);
      mbar_init(bar(st.k_empty[s]), 2);
    }
    for (int s = 0; s < kVStages; ++s) {
      mbar_init(bar(st.v_full[s]), 1);
      mbar_init(bar(st.v_empty[s]), 2);
    }
    for (int x = 0; x < 2; ++x) {
      mbar_init(bar(st.s_full[x]), 1);
      mbar_init(bar(st.s_free[x]), 4);
      mbar_init(bar(st.p_full[x]), 4);
      mbar_init(bar(st.o_ready[x]), 1);
      mbar_init(bar(st.o_free[x]), 4);
      mbar_init(bar(st.part_full[x]), 1);
      mbar_init(bar(st.part_empty[x]), 8 + 2);
      mbar_init(bar(st.drain[x]), 1);
    }
    mbar_init(bar(st.xch_full), 4);
    mbar_init(bar(st.xch_empty), 4);
    st.abort_flag = 0;
    fence_barrier_init();
  }
  __syncthreads();
  const int64_t total = prefix[B];
  const int64_t even = (total + gridDim.x - 1) / gridDim.x;
  const int64_t quota = even > kMinQuota ? even : kMinQuota;
  if (blockIdx.x == 0) {  // for the merge
    for (int r = threadIdx.x; r <= B; r += kTreeThreads) p.plan[1 + r] = prefix[r];
    if (threadIdx.x == 0) p.plan[0] = total > 0 ? quota : 0;
  }
  const int64_t u0 = (int64_t)blockIdx.x * quota, u1 = min(u0 + quota, total);
  if (u0 >= u1) return;  // uniform over the CTA
  if (warp == kIssueWarpA) {
    tmem_alloc(smem_addr(&st.tmem_base), kTmemCols);
    tmem_relinquish();
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = st.tmem_base;

  if (warp == kProducerWarpK || warp == kProducerWarpV) {
    // ------------------------------------------------------------ producers
    // Both walk the CTA's parts; the K producer also hands them out and loads
    // the query tiles. Two warps, because the issue of a block's 16 boxes by
    // one took longer than their transfer.
    const bool is_k = warp == kProducerWarpK;
    if (lane == 0) {
      prefetch_tensormap(is_k ? &kmap : &vmap);
      prefetch_tensormap(&qmap);
      prefetch_tensormap(&qmap_alt);
    }
    // one pass over the cache, re-read only by the row's other tiles
    const uint64_t pol = policy_evict_last();
    const uint32_t ring = is_k ? sK : sV, stages = is_k ? kKStages : kVStages;
    const CUtensorMap* map = is_k ? &kmap : &vmap;
    uint64_t* full = is_k ? st.k_full : st.v_full;
    uint64_t* empty = is_k ? st.k_empty : st.v_empty;
    uint32_t kv_it = 0, q_issued = 0;
    int row = 0;
    {
      int lo = 0, hi = B;  // prefix[lo] <= u0 < prefix[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (prefix[mid] <= u0) lo = mid; else hi = mid;
      }
      row = lo;
    }
    RowGeom w;
    int32_t ignored = 0;
    row_geom(p, row, &w, &ignored);
    int64_t off = u0 - prefix[row];
    int kvh = (int)(off / w.head_cost());
    off -= kvh * w.head_cost();
    int tile = (int)min(off / w.pair_cost, (int64_t)(w.tiles - 1));
    int64_t u = u0 - (off - tile * w.pair_cost);  // start of the current item on the line
    for (int i = 0;;) {
      // the next part with blocks in [u0, u1)
      Part a;
      a.row = -1;
      while (u < u1) {
        const int64_t cost = tile < w.tiles - 1 ? w.pair_cost : w.last_cost;
        a.b0 = blocks_before(u0 - u, w.nb, cost);
        a.b1 = blocks_before(u1 - u, w.nb, cost);
        if (a.b0 < a.b1) {
          const int tile_tok = kItemRows / g;
          a.row = row;
          a.node = tile * tile_tok;
          a.token = w.q0 + a.node;
          a.n_tok = min(tile_tok, w.L - a.node);
          a.ctx = w.C;
          a.len = w.S;
          a.kvh = kvh;
          a.kb0 = w.kb0;
          a.key_begin = w.key_begin;
          a.slot = a.b0 == 0 && a.b1 == w.nb ? -1 : 2 * (int)blockIdx.x + (a.b0 == 0 ? 1 : 0);
          a.alt = a.n_tok * g <= kTileRows;
        }
        u += cost;
        if (++tile == w.tiles) {
          tile = 0;
          if (++kvh == Hkv) {
            kvh = 0;
            do ++row;
            while (row < B && prefix[row + 1] == prefix[row]);
            if (row < B) row_geom(p, row, &w, &ignored);
          }
        }
        if (a.row >= 0) break;
      }
      if (is_k) {
        const int slot = i & 1;
        if (i >= 2 && !__all_sync(0xffffffffu, wait_sleep(bar(st.part_empty[slot]), ((i >> 1) - 1) & 1, abort_flag)))
          break;
        if (lane == 0) {
          st.parts[slot] = a;
          mbar_arrive(bar(st.part_full[slot]));
        }
      }
      if (a.row < 0) break;
      const int* bt_row = p.block_table + (size_t)a.row * p.max_pages;
      const int pg0 = a.kb0 / kPage + a.b0 * kBlockPages;
      const int page_end = (a.len + kPage - 1) / kPage;
      auto load_ids = [&](int c) -> int {  // page id of page pg0 + 32c + lane, or -1
        const int lp = pg0 + 32 * c + lane;
        int v = -1;
        if (lp < page_end && lp < pg0 + (a.b1 - a.b0) * kBlockPages) {
          v = __ldg(bt_row + lp);
          if (v < 0 || v >= p.num_pages) {
            atomicOr(p.status, kStatusBadPage);
            v = -1;
          }
        }
        return v;
      };
      int ids = load_ids(0), ids_next = load_ids(1);
      if (is_k) {
        if (i >= 1 && !__all_sync(0xffffffffu, wait_sleep(bar(st.q_empty), (i - 1) & 1, abort_flag))) break;
        if (lane == 0) {
          mbar_arrive_expect_tx(bar(st.q_full), a.alt ? kTileQBytes : kQBytes);
          tma_load_3d(sQ, a.alt ? &qmap_alt : &qmap, 0, a.kvh * g, a.token, bar(st.q_full));
        }
        q_issued = i + 1;
      }
      ++i;
      bool ok = true;
      const int n = a.b1 - a.b0;
      for (int b = 0; b < n; ++b, ++kv_it) {
        if (b > 0 && (b * kBlockPages) % 32 == 0) {
          ids = ids_next;
          ids_next = load_ids(b * kBlockPages / 32 + 1);
        }
        const uint32_t s = kv_it % stages;
        if (kv_it >= stages) {
          ok = __all_sync(0xffffffffu, wait_sleep(bar(empty[s]), (kv_it / stages - 1) & 1, abort_flag));
          if (!ok) break;
        }
        arrive_expect_tx_e(bar(full[s]), kBlockBytes);
#pragma unroll
        for (int j = 0; j < kBlockPages; ++j) {
          const int pid = __shfl_sync(0xffffffffu, ids, (b * kBlockPages) % 32 + j);
          const int y = pid < 0 ? p.oob_row : (pid * Hkv + a.kvh) * kPage;
          tma_load_2d_e(ring + s * kBlockBytes + j * kTileBytes, map, y, bar(full[s]), pol);
        }
      }
      if (!ok) break;
    }
    // after an abort: wait (bounded) for the copies still in flight
    if (*abort_flag && lane == 0) {
      for (uint32_t it = kv_it > stages ? kv_it - stages : 0; it < kv_it; ++it)
        mbar_wait(bar(full[it % stages]), (it / stages) & 1);
      if (q_issued > 0) mbar_wait(bar(st.q_full), (q_issued - 1) & 1);
    }
  } else if (warp == kIssueWarpA || warp == kIssueWarpA + 1) {
    // ---------------------------------------------------------- MMA issuers
    constexpr uint32_t idS = idesc_bf16(kTileRows, kBlockKeys, false, false);
    constexpr uint32_t idO = idesc_bf16(kTileRows, kHeadDim, false, true);
    constexpr uint64_t kStageStep = kBlockBytes / 16, kVStep = 16 * kRowBytes / 16;
    const uint64_t kdesc0 = smem_desc_sw128(sK, 16, 1024), vdesc0 = smem_desc_sw128(sV, 1024, 1024);
    const int x = warp - kIssueWarpA;
    const uint32_t scol = tmem + col_s(x), pcol = tmem + col_p(x), ocol = tmem + col_o(x);
    uint32_t kv_it = 0, cnt = 0;  // blocks of the CTA, blocks of this tile, before the part
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int slot = i & 1;
      if (!wait_sleep(bar(st.part_full[slot]), (i >> 1) & 1, abort_flag)) break;
      const Part a = st.parts[slot];
      if (a.row < 0) break;
      if (!wait_sleep(bar(st.q_full), i & 1, abort_flag)) break;
      const int n = a.b1 - a.b0;
      const int nx = a.alt ? (n + 1 - x) / 2 : n;  // this tile's blocks: x, x + 2, ... or all
      const uint64_t qd = smem_desc_sw128(sQ + (a.alt ? 0 : x) * kTileQBytes, 16, 1024);
      if (nx == 0) tc_commit_e(bar(st.q_empty));
      for (int b = 0; b <= nx && nx > 0; ++b) {
        if (b < nx) {  // S(b)
          const uint32_t it = kv_it + (a.alt ? 2 * b + x : b), bk = cnt + b;
          const int s = it % kKStages;
          if (!wait_sleep(bar(st.k_full[s]), (it / kKStages) & 1, abort_flag) ||
              (bk >= 1 && !wait_sleep(bar(st.s_free[x]), (bk - 1) & 1, abort_flag))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t kd = kdesc0 + s * kStageStep;
          tc_mma_ss_e(scol, qd, kd, idS, 0u);
#pragma unroll
          for (int kk = 1; kk < kHeadDim / 16; ++kk)
            tc_mma_ss_e(scol, qd + (uint64_t)(kk * 2), kd + (uint64_t)(kk * 2), idS, 1u);
          tc_commit_e(bar(st.s_full[x]));
          tc_commit_e(bar(st.k_empty[s]));
          if (a.alt) tc_commit_e(bar(st.k_empty[s]));  // the other tile does not read this stage
          if (b == nx - 1) tc_commit_e(bar(st.q_empty));
        }
        if (b >= 1) {  // O += P(b - 1) V(b - 1)
          const uint32_t it = kv_it + (a.alt ? 2 * (b - 1) + x : b - 1), bk = cnt + b - 1;
          const int s = it % kVStages;
          if (!wait_sleep(bar(st.v_full[s]), (it / kVStages) & 1, abort_flag) ||
              !wait_sleep(bar(st.p_full[x]), bk & 1, abort_flag) ||
              (b == 1 && i >= 1 && !wait_sleep(bar(st.o_free[x]), (i - 1) & 1, abort_flag))) {
            ok = false;
            break;
          }
          tc_fence_after();
          const uint64_t vd = vdesc0 + s * kStageStep;
          tc_mma_ts_e(ocol, pcol, vd, idO, b > 1 ? 1u : 0u);
#pragma unroll
          for (int kk = 1; kk < kBlockKeys / 16; ++kk) tc_mma_ts_e(ocol, pcol + kk * 8, vd + kk * kVStep, idO, 1u);
          tc_commit_e(bar(st.o_ready[x]));
          tc_commit_e(bar(st.v_empty[s]));
          if (a.alt) tc_commit_e(bar(st.v_empty[s]));
        }
      }
      if (!ok) break;
      cnt += nx;
      kv_it += n;
      if (lane == 0) mbar_arrive(bar(st.part_empty[slot]));
    }
    // MMAs still in flight (after an abort) must not outlive TMEM
    tc_commit_e(bar(st.drain[x]));
    mbar_wait(bar(st.drain[x]), 0);
  } else {
    // -------------------------------------------------------------- softmax
    const int x = warp >> 2, wq = warp & 3;
    const int row = threadIdx.x & (kTileRows - 1);
    const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
    const uint32_t cS = tmem + lane_off + col_s(x), cP = tmem + lane_off + col_p(x), cO = tmem + lane_off + col_o(x);
    const int tok0 = row / g, head = row % g;
    uint32_t kv_it = 0, cnt = 0, n_xch = 0;
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int slot = i & 1;
      ok = __all_sync(0xffffffffu, wait_poll(bar(st.part_full[slot]), (i >> 1) & 1, abort_flag));
      if (!ok) break;
      const Part& a = st.parts[slot];  // valid until part_empty; re-read where needed to save registers
      if (a.row < 0) break;
      const bool alt = a.alt;
      const int n = a.b1 - a.b0;
      const int nx = alt ? (n + 1 - x) / 2 : n;
      const int tok = (alt ? 0 : x * (kTileRows / g)) + tok0;
      const bool busy = (alt ? 0 : x * kTileRows) + wq * 32 < a.n_tok * g;  // this warp has rows
      const int t = a.token + min(tok, a.n_tok - 1);
      int lo = 0;
      if (p.window > 0) lo = min(max(__ldg(p.positions + t), a.ctx), a.len - 1) - p.window + 1;
      // blocks that need no mask: keys [plain_lo, ctx) are seen by every node
      const int plain_lo = p.window > 0 ? a.len - p.window : 0, plain_hi = a.ctx - kBlockKeys;
      int kb = a.kb0 + (a.b0 + (alt ? x : 0)) * kBlockKeys;
      uint32_t it = kv_it + (alt ? x : 0);
      float m_ref = -INFINITY, l = 0.f;
      // V rows that no node sees may hold anything, and a zero weight does not
      // cancel a NaN: they are cleared before the tile's PV reads them
      auto clear_dead = [&](bool dead) -> bool {
        if (!__any_sync(0xffffffffu, dead)) return true;
        const uint32_t s = it % kVStages;
        if (!__all_sync(0xffffffffu, wait_poll(bar(st.v_full[s]), (it / kVStages) & 1, abort_flag))) return false;
        if (dead) {
#pragma unroll
          for (int c = 0; c < 8; ++c) zero_smem16(sV + s * kBlockBytes + row * kRowBytes + c * 16);
        }
        fence_proxy_async();
        return true;
      };
      const int kb_step = alt ? 2 * kBlockKeys : kBlockKeys;
      if (!busy) {  // none of this warp's rows is a query: it only keeps the barriers and clears V rows
        for (int b = 0; b < nx; ++b, ++cnt, kb += kb_step, it += alt ? 2 : 1) {
          uint32_t seen[4];
          const bool dead = (kb > plain_hi || kb < plain_lo) && block_masks(p, a, t, lo, kb, wq, lane, seen);
          ok = __all_sync(0xffffffffu, wait_poll(bar(st.s_full[x]), cnt & 1, abort_flag));
          if (!ok) break;
          if (lane == 0) mbar_arrive(bar(st.s_free[x]));
          // in step with the other warps: one arrival per phase
          if (cnt >= 1) {
            ok = __all_sync(0xffffffffu, wait_poll(bar(st.o_ready[x]), (cnt - 1) & 1, abort_flag));
            if (!ok) break;
          }
          ok = clear_dead(dead);
          if (!ok) break;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(st.p_full[x]));
        }
      } else {
        for (int b = 0; b < nx; ++b, ++cnt, kb += kb_step, it += alt ? 2 : 1) {
          const bool masked = kb > plain_hi || kb < plain_lo;
          uint32_t seen[4];  // bit e of word c: this thread's node sees key kb + 32c + e
          bool dead = false;
          if (masked) dead = block_masks(p, a, t, lo, kb, wq, lane, seen);
          ok = __all_sync(0xffffffffu, wait_poll(bar(st.s_full[x]), cnt & 1, abort_flag));
          if (!ok) break;
          tc_fence_after();
          uint32_t sv[2][32], pk[32];
          tmem_ld32(cS, sv[0]);
          tmem_ld32(cS + 32, sv[1]);
          tmem_ld_wait();
          if (masked) {
            hide(sv[0], seen[0]);
            hide(sv[1], seen[1]);
          }
          float alpha = 1.f;
          float l0 = chunk_weights(sv, p.scale_log2, m_ref, alpha, pk);
          // the P buffer was last read by the tile's previous PV
          if (cnt >= 1) {
            ok = __all_sync(0xffffffffu, wait_poll(bar(st.o_ready[x]), (cnt - 1) & 1, abort_flag));
            if (!ok) break;
            tc_fence_after();
          }
          tmem_st32(cP, pk);
          tmem_ld32(cS + 64, sv[0]);
          tmem_ld32(cS + 96, sv[1]);
          tmem_ld_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(st.s_free[x]));
          if (masked) {
            hide(sv[0], seen[2]);
            hide(sv[1], seen[3]);
          }
          float a1 = 1.f;
          const float l1 = chunk_weights(sv, p.scale_log2, m_ref, a1, pk);
          if (__any_sync(0xffffffffu, a1 != 1.f)) {  // the reference rose: rescale the first half's weights too
            tmem_st_wait();
            uint32_t pv[32];
            tmem_ld32(cP, pv);
            tmem_ld_wait();
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float2 f = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&pv[e]));
              pv[e] = pack_bf16x2(f.x * a1, f.y * a1);
            }
            tmem_st32(cP, pv);
            l0 *= a1;
            alpha *= a1;
          }
          tmem_st32(cP + 32, pk);
          l = l * alpha + (l0 + l1);
          ok = clear_dead(dead);
          if (!ok) break;
          if (b > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
            uint32_t ov[32];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              tmem_ld32(cO + 32 * h, ov);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * alpha);
              tmem_st32(cO + 32 * h, ov);
            }
          }
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(st.p_full[x]));
        }
      }
      if (!ok) break;
      kv_it += n;
      // ---- end of the part
      if (nx > 0) {
        ok = __all_sync(0xffffffffu, wait_poll(bar(st.o_ready[x]), (cnt - 1) & 1, abort_flag));
        if (!ok) break;
      }
      tc_fence_after();
      uint32_t ov[2][32];
      if (busy && nx > 0) {
        tmem_ld32(cO, ov[0]);
        tmem_ld32(cO + 32, ov[1]);
        tmem_ld_wait();
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) ov[0][e] = ov[1][e] = 0u;
      }
      const int token = a.token, kvh = a.kvh, part_slot = a.slot;
      bool writes = tok < a.n_tok;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(st.o_free[x]));
        mbar_arrive(bar(st.part_empty[slot]));
      }
      if (alt) {  // tile B hands its state to tile A
        const uint32_t ph = n_xch & 1;
        if (x == 1) {
          if (n_xch >= 1) {
            ok = __all_sync(0xffffffffu, wait_poll(bar(st.xch_empty), ph ^ 1, abort_flag));
            if (!ok) break;
          }
          if (busy) {
#pragma unroll
            for (int d = 0; d < kHeadDim; ++d) xch[d * kTileRows + row] = __uint_as_float(ov[d >> 5][d & 31]);
            xch[kHeadDim * kTileRows + row] = m_ref;
            xch[(kHeadDim + 1) * kTileRows + row] = l;
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(st.xch_full));
          writes = false;
        } else {
          ok = __all_sync(0xffffffffu, wait_poll(bar(st.xch_full), ph, abort_flag));
          if (!ok) break;
          if (busy) {
            const float mb = xch[kHeadDim * kTileRows + row], lb = xch[(kHeadDim + 1) * kTileRows + row];
            const float M = fmaxf(m_ref, mb);
            const float fa = m_ref > -INFINITY ? exp2f(m_ref - M) : 0.f, fb = mb > -INFINITY ? exp2f(mb - M) : 0.f;
            l = l * fa + lb * fb;
            m_ref = M;
#pragma unroll
            for (int d = 0; d < kHeadDim; ++d)
              ov[d >> 5][d & 31] = __float_as_uint(__uint_as_float(ov[d >> 5][d & 31]) * fa + xch[d * kTileRows + row] * fb);
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(st.xch_empty));
        }
        ++n_xch;
      }
      if (writes) {
        float inv = l > 0.f ? 1.f / l : 0.f;
        float lse2 = l > 0.f ? m_ref + __log2f(l) : -INFINITY;
        const int h = kvh * g + head;
        if (part_slot < 0) {
          if (p.sinks != nullptr) inv = finish_with_sink(m_ref, l, tree_sink(p, h), &lse2);
          const size_t orow = (size_t)(token + tok) * Hq + h;
          uint4* dst = reinterpret_cast<uint4*>(p.out + orow * kHeadDim);
#pragma unroll
          for (int v = 0; v < 8; ++v) {
            const int hh = v >> 2, e0 = (v & 3) * 8;
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
              o[k] = pack_bf16x2(__uint_as_float(ov[hh][e0 + 2 * k]) * inv, __uint_as_float(ov[hh][e0 + 2 * k + 1]) * inv);
            dst[v] = make_uint4(o[0], o[1], o[2], o[3]);
          }
          p.lse[orow] = lse2 * 0.69314718055994531f;
        } else {
          const size_t prow = (size_t)part_slot * kItemRows + (alt ? 0 : x * kTileRows) + row;
          float4* dst = reinterpret_cast<float4*>(p.o_part + prow * kHeadDim);
#pragma unroll
          for (int v = 0; v < 16; ++v) {
            const int hh = v >> 3, e0 = (v & 7) * 4;
            dst[v] = make_float4(__uint_as_float(ov[hh][e0]) * inv, __uint_as_float(ov[hh][e0 + 1]) * inv,
                                 __uint_as_float(ov[hh][e0 + 2]) * inv, __uint_as_float(ov[hh][e0 + 3]) * inv);
          }
          p.lse_part[prow] = lse2;
        }
      }
    }
  }

  __syncwarp();
  if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, kStatusTimeout);
  tc_fence_before();
  __syncthreads();
  if (warp == kIssueWarpA) {
    tc_fence_after();
    tmem_dealloc(tmem, kTmemCols);
  }
}

// Joins the parts of items that cross a cut of the line: out = sum_i 2^(b_i - b) o_i,
// b = log2 sum_i 2^(b_i), in the order of the CTAs. One warp per (token, q
// head), two dims a lane; heads of unsplit items leave at once.
constexpr int kMergeWarps = 8;

__global__ void __launch_bounds__(kMergeWarps * 32) merge_tree_kernel(const TreeParams p) {
  grid_dep_wait();
  const int64_t quota = p.plan[0];
  if (quota == 0) return;
  const int64_t* prefix = p.plan + 1;
  const int lane = threadIdx.x & 31, Hq = p.num_q_heads, g = p.group;
  const int64_t n = (int64_t)p.total_q * Hq;
  for (int64_t v = (int64_t)blockIdx.x * kMergeWarps + (threadIdx.x >> 5); v < n; v += (int64_t)gridDim.x * kMergeWarps) {
    const int t = (int)(v / Hq), h = (int)(v % Hq);
    int lo = 0, hi = p.num_seqs;  // qsl[lo] <= t < qsl[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (__ldg(p.qsl + mid) <= t) lo = mid; else hi = mid;
    }
    RowGeom w;
    int32_t ignored = 0;
    if (!row_geom(p, lo, &w, &ignored) || t < w.q0 || t >= w.q0 + w.L) continue;
    const int tile_tok = kItemRows / g, tile = (t - w.q0) / tile_tok;
    const int64_t cost = tile < w.tiles - 1 ? w.pair_cost : w.last_cost;
    const int64_t u = prefix[lo] + (h / g) * w.head_cost() + tile * w.pair_cost;
    const int c0 = (int)(u / quota), c1 = (int)((u + cost - 1) / quota);
    const int prow = (t - w.q0 - tile * tile_tok) * g + h % g;
    // parts of CTA c: blocks [before(c), before(c + 1))
    float bmax = tree_sink(p, h);
    const float s2 = bmax;
    bool split = false;
    for (int c = c0; c <= c1; ++c) {
      const int b0 = blocks_before((int64_t)c * quota - u, w.nb, cost);
      const int b1 = blocks_before((int64_t)(c + 1) * quota - u, w.nb, cost);
      if (b0 == b1) continue;
      if (b0 == 0 && b1 == w.nb) break;  // one part, written by its CTA
      split = true;
      bmax = fmaxf(bmax, p.lse_part[(size_t)(2 * c + (b0 == 0 ? 1 : 0)) * kItemRows + prow]);
    }
    if (!split) continue;
    float sum = s2 > -INFINITY ? exp2f(s2 - bmax) : 0.f, o0 = 0.f, o1 = 0.f;
    if (bmax > -INFINITY) {
      for (int c = c0; c <= c1; ++c) {
        const int b0 = blocks_before((int64_t)c * quota - u, w.nb, cost);
        const int b1 = blocks_before((int64_t)(c + 1) * quota - u, w.nb, cost);
        if (b0 == b1) continue;
        const size_t pr = (size_t)(2 * c + (b0 == 0 ? 1 : 0)) * kItemRows + prow;
        const float wt = exp2f(p.lse_part[pr] - bmax);
        const float2 o = reinterpret_cast<const float2*>(p.o_part + pr * kHeadDim)[lane];
        sum += wt;
        o0 += wt * o.x;
        o1 += wt * o.y;
      }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    const size_t orow = (size_t)t * Hq + h;
    reinterpret_cast<uint32_t*>(p.out + orow * kHeadDim)[lane] = pack_bf16x2(o0 * inv, o1 * inv);
    if (lane == 0) p.lse[orow] = sum > 0.f ? (bmax + __log2f(sum)) * 0.69314718055994531f : -INFINITY;
  }
}

}  // namespace

cudaError_t launch_tree(const CUtensorMap& kmap, const CUtensorMap& vmap, const CUtensorMap& qmap,
                        const CUtensorMap& qmap_alt, const TreeParams& p, int sms, cudaStream_t stream) {
  const int grid = sms < kTreeMaxCtas ? sms : kTreeMaxCtas;
  tree_kernel<<<grid, kTreeThreads, tree_smem_bytes(), stream>>>(kmap, vmap, qmap, qmap_alt, p);
  cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess) return e;
  const int64_t heads = (int64_t)p.total_q * p.num_q_heads;
  const int64_t want = (heads + kMergeWarps - 1) / kMergeWarps;
  LaunchCfg lc(dim3((unsigned)(want < sms * 8 ? want : sms * 8)), dim3(kMergeWarps * 32), 0, stream, true);
  return cudaLaunchKernelEx(&lc.cfg, merge_tree_kernel, p);
}

cudaError_t prepare_tree_kernels() {
  const cudaError_t e =
      cudaFuncSetAttribute(tree_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tree_smem_bytes());
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(tree_kernel, cudaFuncAttributePreferredSharedMemoryCarveout,
                              cudaSharedmemCarveoutMaxShared);
}

}  // namespace mcpu
