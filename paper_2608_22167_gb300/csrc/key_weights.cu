// Attention weights per cached key (mcpu_accumulate_weights) on the
// 5th-generation tensor cores:
//   w_j = decay w_j [j < C] + sum_{i: j <= p_i, p_i - j < W} sum_u exp(scale q_iu . k_j - lse_iu)
//
// The keys are the rows of the product: S = K Q^T with 128 keys in TMEM's
// lanes, so that a thread owns a key and the sum over queries stays in its
// registers; with the log-sum-exps given there is no maximum to carry and
// nothing to exchange. A unit is 256 keys (two tiles over one stream of
// queries, which halves its traffic from L2) of one (row, kv head); it walks
// the row's queries in blocks of 128 columns (128 / g queries x g heads), those
// that see some of its keys.
//
// Work: units lie on a line, each weighing 2 and each block 2 more (a unit
// whose queries fit 32 columns weighs 3: there the keys' way from HBM counts);
// the line is cut into equal pieces, one per CTA. A unit of more than
// kWholeBlocks blocks may be cut between blocks: its parts are summed by
// merge_weights_kernel in the order of the pieces. Every CTA derives the line
// from the lengths itself: no planning launch.
//
// Warps: 0 walks the line and brings the keys (TMA, one box per page), 1 issues
// the MMAs, 2 brings the earlier weights, 4-6 bring the queries (one box for 128
// contiguous columns, else 16 bytes a lane, which also gathers the queries of a
// path) and their log-sum-exps, 8-15 and 16-23 take the exponentials, blocks in turn (a warp's
// waits and loads are the other group's work). TMEM: two buffers of 128 columns
// for each half of a unit's keys.
//
// Bound by the keys' way from HBM where queries are few (64 rows of 2047 to 16383
// keys, 64 / 8 heads, one query each: 642 MB in 105 us, 90 % of the copy rate).
// Where they are many, 1024 of a block's 1540 cycles are exponentials, 8 a clock
// and sub-partition; the stall counted most is the wait for loads, and a warp waits
// for its TMEM loads before it uses them (16 rows of 4096 to 32768 keys, 64 to 2048
// queries: 3.2 ms, at 1.95 to 2.07 GHz and below the power limit). There the log-sum-exps as a step of the
// product took 4.55 ms to 3.56: read for every column from shared memory they needed
// 128 bytes a clock; and one box for 128 contiguous columns, not 16 bytes a lane,
// 4.43 to 3.22.
#include "keep.cuh"
#include "warp_pipe.cuh"

namespace mcpu {

namespace {

constexpr int kTileKeys = kBlockKeys, kUnitKeys = 2 * kTileKeys, kCols = 128;
constexpr int kStageBytes = 2 * kBlockBytes, kQBytes = kCols * kRowBytes;
constexpr int kKStages = 4, kQStages = 3, kOldStages = 8, kUnits = 4;
constexpr int kQueryWarps = 3;
// each fills a stage of its own: a warp that came to another's stage two turns
// early would take an older phase of the same parity for its own
static_assert(kQueryWarps == kQStages, "a stage each");
constexpr int kThreads = 768, kGroupWarps = 8;  // warps that take the exponentials of a block
constexpr uint32_t kTmemCols = 512;
// Units of up to so many blocks are never cut, and rows of no more need no merge
// (up to 8: pieces differ too much, the many queries above 3.41 ms, 3 or 1: 3.22).
constexpr int kWholeBlocks = 3;
constexpr int kCostShort = 3;  // of a unit of a row with one block of queries (2 to 4: +-1 %)
constexpr int kMinQuota = 3;   // of a piece: a unit (four rows of 16 to 299 keys: 13 us, at 12 17)
// A fifth step of the product, over 16 dims of which three are used: 1 for every
// key, and -lse / scale of a column in three bf16 pieces (24 bits). As 8 x 16
// byte matrices without swizzle: first dims 0-7 of all rows, then 8-15.
constexpr int kExtraHalf = kCols * 16, kExtraBytes = 2 * kExtraHalf;
constexpr int kRingBytes = kKStages * kStageBytes + kQStages * (kQBytes + kExtraBytes) + kExtraBytes;

struct alignas(16) Unit {
  int32_t row;  // -1: no more units
  int32_t kvh, k0, len, n, q0;  // first key, row length, queries, first query token
  int32_t b0, b1;               // query blocks to do here (none: old weights only decay)
  int32_t slot;                 // partial slot, or -1: the whole unit
  int32_t pairs;                // a run of units with the same one block of queries
};

struct WeightsSmem {
  uint64_t unit_full[kUnits], unit_empty[kUnits];
  uint64_t k_full[kKStages], k_empty[kKStages], q_full[kQStages], q_empty[kQStages];
  uint64_t s_full[2][2], s_empty[2][2];  // [tile][buffer]
  uint64_t old_full[kOldStages], old_empty[kOldStages];
  uint64_t sum_full[kGroupWarps], sum_empty[kGroupWarps];
  uint64_t drain;
  Unit units[kUnits];
  uint32_t pages[kKStages];  // which of a unit's 16 pages exist
  float old[kOldStages][kUnitKeys];  // earlier weights
  float sums[kUnitKeys];             // the second group's, for the first
  int64_t scan[kThreads / 32];
  int64_t prefix[kMaxSeqs + 1];  // cost of the rows before each
  uint32_t tmem_base;
  int32_t abort_flag;
};

size_t weights_smem_bytes() { return 1024 + kRingBytes + sizeof(WeightsSmem); }

// ------------------------------------------------------------ the work line
struct RowGeom {
  int q0, L, S, n, C, window;  // window 0: none that matters
  int tok;                     // queries of a block
  int nb;                      // blocks of all its queries
  int u0, u1;                  // units

  // the blocks of unit u whose queries see some key of it
  __device__ __forceinline__ void blocks(int u, int* b0, int* b1) const {
    const int k0 = u * kUnitKeys, last = min(k0 + kUnitKeys, S) - 1;
    const int i0 = max(0, k0 - C);
    const int i1 = window > 0 ? (int)min((int64_t)n, (int64_t)last - C + window) : n;
    *b0 = i0 / tok;
    *b1 = i1 > i0 ? (i1 + tok - 1) / tok : *b0;
  }
  __device__ __forceinline__ int cost(int u) const {
    int b0, b1;
    blocks(u, &b0, &b1);
    return b1 == b0 ? 1 : nb == 1 ? kCostShort : 2 + 2 * (b1 - b0);
  }
};

// Geometry of row r; false if it has no work, with the status bits of what is wrong.
__device__ __forceinline__ bool row_geom(const WeightParams& p, int r, RowGeom* w, int32_t* bits) {
  w->q0 = p.qsl[r];
  w->L = p.qsl[r + 1] - w->q0;
  w->S = p.seq_lens[r];
  w->n = p.path ? p.path_len[r] : w->L;
  if (w->q0 < 0 || w->L < 0 || w->L > p.total_q - w->q0 || w->n < 0 || w->n > w->S ||
      (p.path && w->n > p.max_path) || w->S > p.max_pages * kPage || w->S > p.max_slots) {
    *bits |= kStatusBadLengths;
    return false;
  }
  if (w->n == 0) return false;
  w->C = w->S - w->n;
  w->window = p.window >= w->S ? 0 : p.window;
  w->tok = kCols / p.group;
  w->nb = (w->n + w->tok - 1) / w->tok;
  // weights before the first window change only if they decay
  w->u0 = w->window > 0 && p.decay == 1.f ? max(0, w->C - w->window + 1) / kUnitKeys : 0;
  w->u1 = (w->S + kUnitKeys - 1) / kUnitKeys;
  return true;
}

// Whether a row's path names queries of the row.
__device__ __forceinline__ bool path_ok(const WeightParams& p, int r, const RowGeom& w) {
  if (!p.path) return true;
  const int32_t* path = p.path + (size_t)r * p.max_path;
  bool ok = true;
#pragma unroll 8
  for (int i = 0; i < w.n; ++i) {
    const int x = path[i];
    ok &= x >= 0 && x < w.L;
  }
  return ok;
}

// Cost of one kv head of the row.
__device__ __forceinline__ int64_t head_cost(const RowGeom& w) {
  int64_t sum = 0;
  int u = w.u0;
  if (w.window == 0) {  // all blocks see the keys before the first query
    const int all = min(w.u1, (w.C + w.tok - 1) / kUnitKeys + 1);
    sum = (int64_t)(w.nb == 1 ? kCostShort : 2 + 2 * w.nb) * all;
    u = all;
  }
  for (; u < w.u1; ++u) sum += w.cost(u);
  return sum;
}

// Blocks of a unit that belong to the pieces ending x units of cost into it.
__device__ __forceinline__ int blocks_before(int64_t x, int nb) {
  if (nb <= kWholeBlocks) return x <= 0 ? 0 : nb;
  return x <= 2 ? 0 : x >= 2 + 2 * nb ? nb : (int)((x - 1) / 2);
}

__device__ __forceinline__ bool unit_ok(const WeightParams& p, const Unit& a) {
  return a.row < p.num_seqs && a.kvh >= 0 && a.kvh < p.num_kv_heads && a.k0 >= 0 && a.k0 < a.len &&
         a.len <= p.max_slots && a.n >= 1 && a.n <= a.len && a.b0 >= 0 && a.b1 >= a.b0 &&
         (int64_t)(a.b1 - 1) * (kCols / p.group) < a.n && a.q0 >= 0 && a.q0 < p.total_q && a.slot < 2 * kWeightCtas && a.pairs >= 1 &&
         (int64_t)a.k0 + (int64_t)(a.pairs - 1) * kUnitKeys < a.len && (a.pairs == 1 || a.b1 == a.b0 + 1);
}

// Descriptor of the fifth step's operands.
__device__ __forceinline__ uint64_t extra_desc(uint32_t saddr) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(kExtraHalf >> 4) << 16 | (uint64_t)(128 >> 4) << 32 |
         (uint64_t)1 << 46;
}

// S = K Q^T - lse / scale of one tile by one elected lane of a warp in step, and the commit behind it.
__device__ __forceinline__ void mma_keys_e(uint32_t d, uint64_t k, uint64_t q, uint64_t ones, uint64_t lse,
                                           uint32_t idesc, uint32_t done) {
  static_assert(kHeadDim == 64, "four steps of 16 dims, 32 bytes each");
  asm volatile(
      "{\n\t.reg .pred e, t, f;\n\t.reg .b64 a, b;\n\telect.sync _|e, 0xffffffff;\n\t"
      "setp.eq.u32 t, 0, 0;\n\tsetp.ne.u32 f, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, f;\n\t"
      "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
      "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
      "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %5, %6, %3, t;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n\t"
      "}" ::"r"(d),
      "l"(k), "l"(q), "r"(idesc), "r"(done), "l"(ones), "l"(lse)
      : "memory");
}

// One word from global to shared memory, asynchronously; the arrival of this
// thread on a barrier once all its copies so far have landed; the wait for them.
__device__ __forceinline__ void copy_word(uint32_t dst, const float* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_arrive(uint32_t bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// Columns of block b of a unit: those of its queries, and rounded up to the MMA's step.
__device__ __forceinline__ int block_cols(const Unit& a, int b, int g) { return min(kCols, (a.n - b * (kCols / g)) * g); }

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[32]) {  // into the first 16
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
        "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
      : "r"(taddr));
#pragma unroll
  for (int e = 16; e < 32; ++e) v[e] = 0u;
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

// Waits for this thread's TMEM loads; what they loaded is not used before.
__device__ __forceinline__ void tmem_ld_wait_for(uint32_t (&v)[32]) {
  tmem_ld_wait();
#pragma unroll
  for (int e = 0; e < 32; ++e) asm volatile("" : "+r"(v[e]));
}

// sum += 2^(s scale) over kN columns; masked: only columns lo <= c < hi.
template <int kN, bool kMasked>
__device__ __forceinline__ void add_columns(const uint32_t (&sv)[32], uint64_t sc, int lo, int hi, uint64_t (&sum)[2]) {
#pragma unroll
  for (int c = 0; c < kN; c += 2) {
    const uint64_t x = mul2((uint64_t)sv[c] | ((uint64_t)sv[c + 1] << 32), sc);
    float x0 = lo_f32(x), x1 = hi_f32(x);
    if (kMasked) {
      x0 = c >= lo && c < hi ? x0 : -INFINITY;
      x1 = c + 1 >= lo && c + 1 < hi ? x1 : -INFINITY;
    }
    sum[(c >> 1) & 1] = add2(sum[(c >> 1) & 1], pack_f32x2(ex2_approx(x0), ex2_approx(x1)));
  }
}

__global__ void __launch_bounds__(kThreads, 1)
    weights_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap qmap,
                   const WeightParams p) {
  extern __shared__ uint8_t smem_raw[];
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - raw);
  WeightsSmem& st = *reinterpret_cast<WeightsSmem*>(base_ptr + kRingBytes);
  volatile int32_t* abort_flag = &st.abort_flag;
  auto bar = [&](uint64_t& b) { return smem_addr(&b); };
  const int B = p.num_seqs, g = p.group, Hkv = p.num_kv_heads, Hq = p.num_q_heads;
  const uint32_t sK = base, sQ = base + kKStages * kStageBytes, sLse = sQ + kQStages * kQBytes,
                 sOnes = sLse + kQStages * kExtraBytes;

  // Before anything is read: TMEM, the barriers, the tensor maps.
  if (warp == 0) {
    tmem_alloc(smem_addr(&st.tmem_base), kTmemCols);
    tmem_relinquish();
  }
  if (threadIdx.x == 32) {
    for (int i = 0; i < kUnits; ++i) {
      mbar_init(bar(st.unit_full[i]), 1);
      mbar_init(bar(st.unit_empty[i]), 1 + 1 + kQueryWarps + 2 * kGroupWarps);
    }
    for (int i = 0; i < kKStages; ++i) {
      mbar_init(bar(st.k_full[i]), 2);
      mbar_init(bar(st.k_empty[i]), 1 + kGroupWarps);
    }
    for (int i = 0; i < kQStages; ++i) {
      mbar_init(bar(st.q_full[i]), 2);
      mbar_init(bar(st.q_empty[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(bar(st.s_full[i >> 1][i & 1]), 1);
      mbar_init(bar(st.s_empty[i >> 1][i & 1]), 4);
    }
    for (int i = 0; i < kOldStages; ++i) {
      mbar_init(bar(st.old_full[i]), 32);
      mbar_init(bar(st.old_empty[i]), kGroupWarps);
    }
    for (int i = 0; i < kGroupWarps; ++i) {
      mbar_init(bar(st.sum_full[i]), 1);
      mbar_init(bar(st.sum_empty[i]), 1);
    }
    mbar_init(bar(st.drain), 1);
    st.abort_flag = 0;
    fence_barrier_init();
  }
  for (int i = threadIdx.x; i < (kQStages + 1) * kExtraBytes / 16; i += kThreads) {
    const bool ones = i >= kQStages * kExtraBytes / 16 && i < (kQStages * kExtraBytes + kExtraHalf) / 16;
    *reinterpret_cast<uint4*>(base_ptr + (sLse - base) + 16 * i) = ones ? make_uint4(0x3f803f80u, 0x3f80u, 0u, 0u)
                                                                        : make_uint4(0u, 0u, 0u, 0u);
  }
  fence_proxy_async();
  if (threadIdx.x == 64) {
    prefetch_tensormap(&kmap);
    prefetch_tensormap(&qmap);
  }
  auto leave = [&] {  // the whole CTA
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
      tc_fence_after();
      tmem_dealloc(st.tmem_base, kTmemCols);
    }
    if (threadIdx.x == 0 && *abort_flag == 1) atomicOr(p.status, kStatusTimeout);
  };
  grid_dep_launch();
  grid_dep_wait();
  if (threadIdx.x == 0) p.cuts[blockIdx.x] = make_int4(-1, 0, 0, 0);
  const bool ends = p.qsl[0] == 0 && p.qsl[B] == p.total_q;
  // ---- the line: prefix[r] = cost of the rows before r
  {
    const int per = (B + kThreads - 1) / kThreads;
    const int r0 = min(B, (int)threadIdx.x * per), r1 = min(B, r0 + per);
    int64_t sum = 0;
    int32_t bits = 0;
    RowGeom w;
    for (int r = r0; r < r1; ++r) {
      st.prefix[r] = sum;
      if (!row_geom(p, r, &w, &bits)) continue;
      if (!path_ok(p, r, w)) {
        bits |= kStatusBadLengths;
        continue;
      }
      sum += head_cost(w) * Hkv;
    }
    if (!ends) bits = threadIdx.x == 0 ? kStatusBadLengths : 0;
    if (bits && blockIdx.x == 0) atomicOr(p.status, bits);
    int64_t incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, (long long)incl, o);
      if (lane >= o) incl += v;
    }
    if (lane == 31) st.scan[warp] = incl;
    __syncthreads();
    int64_t at = incl - sum;
    for (int i = 0; i < warp; ++i) at += st.scan[i];
    for (int r = r0; r < r1; ++r) st.prefix[r] += at;
    if (threadIdx.x == kThreads - 1) st.prefix[B] = at + sum;
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const int64_t total = st.prefix[B];
  const int64_t quota = max((total + gridDim.x - 1) / gridDim.x, (int64_t)kMinQuota);
  const int64_t begin = (int64_t)blockIdx.x * quota, end = min(begin + quota, total);
  if (!ends || begin >= total) return leave();  // uniform over the CTA

  if (warp == 0) {
    // ------------------------------------------------- the line, and the keys
    bool ok = true;
    RingAt<kKStages> rk;
    RingAt<kUnits> ru;
    uint32_t loaded = 0;
    int row = 0;
    for (int r = 1 + lane; r < B; r += 32) row += st.prefix[r] <= begin;
    row = __reduce_add_sync(0xffffffffu, row);  // the last row that begins at or before
    RowGeom w;
    int32_t ignored = 0;
    row_geom(p, row, &w, &ignored);
    const int64_t per_head = (st.prefix[row + 1] - st.prefix[row]) / Hkv;
    const int64_t off = begin - st.prefix[row];
    int kvh = (int)(off / per_head);
    const int64_t rem = off - kvh * per_head;
    int u = w.u0;
    int64_t pos = 0;  // cost of the head's units before u
    for (;; u += 32) {
      int64_t incl = u + lane < w.u1 ? w.cost(u + lane) : 0;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, (long long)incl, o);
        if (lane >= o) incl += v;
      }
      const uint32_t past = __ballot_sync(0xffffffffu, pos + incl > rem);
      if (past || u + 32 >= w.u1) {
        const int k = past ? __ffs(past) - 1 : 0;
        const int64_t before = __shfl_sync(0xffffffffu, (long long)incl, max(k - 1, 0));
        if (k > 0) pos += before;
        u += k;
        break;
      }
      pos += __shfl_sync(0xffffffffu, (long long)incl, 31);
    }
    pos += begin - rem;  // where the unit begins on the line
    // page ids of a row from a unit on, two units' at a time
    auto page_of = [&](int r, int unit) -> int {
      const int64_t lp = (int64_t)unit * (kUnitKeys / kPage) + lane;
      return lp < p.max_pages ? p.block_table[(size_t)r * p.max_pages + lp] : -1;
    };
    int ids = page_of(row, u);
    while (pos < end && ok) {
      int b0, b1;
      w.blocks(u, &b0, &b1);
      const int nb = b1 - b0, c = w.cost(u);
      const int s0 = blocks_before(begin - pos, nb), s1 = blocks_before(end - pos, nb);
      Unit a;
      a.row = row;
      a.kvh = kvh;
      a.k0 = u * kUnitKeys;
      a.len = w.S;
      a.n = w.n;
      a.q0 = w.q0;
      a.b0 = b0 + s0;
      a.b1 = b0 + s1;
      a.slot = s0 == 0 && s1 == nb ? -1 : 2 * (int)blockIdx.x + (s0 == 0 ? 1 : 0);
      a.pairs = 1;
      const bool mine = s1 > s0 || (nb == 0 && begin <= pos);
      // units that begin in this piece, all with the same block of queries
      if (mine && w.nb == 1 && w.window == 0)
        a.pairs = (int)min((int64_t)(w.u1 - u), (end - pos + kCostShort - 1) / kCostShort);
      if (mine && a.slot >= 0 && s0 == 0 && lane == 0) {
        int last = blockIdx.x;
        for (int64_t e = end; blocks_before(e - pos, nb) < nb; e += quota) ++last;
        p.cuts[blockIdx.x] = make_int4(last, row, kvh, a.k0);
      }
      // the next unit
      const int C = w.C, W = w.window;
      int these = ids, next_ids = -1;
      const int second = u + 2;
      pos += (int64_t)c * a.pairs;
      u += a.pairs;
      if (u == w.u1) {
        u = w.u0;
        if (++kvh == Hkv) {
          kvh = 0;
          do ++row;
          while (row < B && st.prefix[row + 1] == st.prefix[row]);
          if (row < B) {
            row_geom(p, row, &w, &ignored);
            u = w.u0;
          }
        }
      }
      if (pos < end) ids = page_of(row, u);
      if (!mine) continue;
      if (!unit_ok(p, a)) {
        atomicOr(p.status, kStatusPlanOverflow);
        *abort_flag = 2;
        ok = false;
        break;
      }
      if (a.pairs > 2) next_ids = page_of(a.row, second);
      ok = wait_warp(bar(st.unit_empty[ru.s]), ru.parity ^ 1);
      if (!ok) break;
      if (lane == 0) {
        st.units[ru.s] = a;
        mbar_arrive(bar(st.unit_full[ru.s]));
      }
      __syncwarp();
      ru.next();
      if (a.b0 == a.b1) continue;
#pragma unroll 1
      for (int i = 0; i < a.pairs; ++i) {
        if (i > 0 && !(i & 1)) {
          these = next_ids;
          if (i + 2 < a.pairs) next_ids = page_of(a.row, second + i);
        }
        const int id = __shfl_sync(0xffffffffu, these, (i & 1) * 16 + (lane & 15));
        const int pk = a.k0 + i * kUnitKeys + (lane & 15) * kPage, pl = min(pk + kPage, a.len) - 1;  // the page's keys
        const bool exists = id >= 0 && id < p.num_pages;
        const bool seen = pk < a.len && (W == 0 || pl >= C || (int64_t)pl + W > C);
        if (seen && !exists && lane < 16) atomicOr(p.status, kStatusBadPage);
        const uint32_t pages = __ballot_sync(0xffffffffu, exists) & 0xffffu;
        const int y = exists && pk < a.len ? (id * Hkv + a.kvh) * kPage : p.oob_row;
        ok = wait_warp(bar(st.k_empty[rk.s]), rk.parity ^ 1);
        if (!ok) break;
        st.pages[rk.s] = pages;
        __syncwarp();
        int ys[kBlockPages];
#pragma unroll
        for (int j = 0; j < kBlockPages; ++j) ys[j] = __shfl_sync(0xffffffffu, y, j);
        load_block_e(sK + rk.s * kStageBytes, &kmap, ys, bar(st.k_full[rk.s]), policy_evict_first());
#pragma unroll
        for (int j = 0; j < kBlockPages; ++j) ys[j] = __shfl_sync(0xffffffffu, y, kBlockPages + j);
        load_block_e(sK + rk.s * kStageBytes + kBlockBytes, &kmap, ys, bar(st.k_full[rk.s]), policy_evict_first());
        rk.next();
        ++loaded;
      }
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
    if (ok && wait_warp(bar(st.unit_empty[ru.s]), ru.parity ^ 1)) {
      if (lane == 0) {  // no more units
        st.units[ru.s].row = -1;
        mbar_arrive(bar(st.unit_full[ru.s]));
      }
    }
    // after an abort: wait (bounded) for the copies still in flight
    if (*abort_flag && lane == 0)
      for (uint32_t k = loaded > kKStages ? loaded - kKStages : 0; k < loaded; ++k)
        mbar_wait(bar(st.k_full[k % kKStages]), (k / kKStages) & 1);
  } else if (warp == 1) {
    // -------------------------------------------------------------- MMA issue
    const uint64_t kdesc0 = smem_desc_sw128(sK, 16, 1024), qdesc0 = smem_desc_sw128(sQ, 16, 1024);
    const uint64_t ldesc0 = extra_desc(sLse), ones = extra_desc(sOnes);
    RingAt<kKStages> rk;
    RingAt<kQStages> rq;
    RingAt<kUnits> ru;
    RingAt<2> rs;
    bool ok = true;
    while (ok) {
      ok = wait_warp(bar(st.unit_full[ru.s]), ru.parity);
      if (!ok) break;
      const Unit a = st.units[ru.s];
      if (a.row < 0) break;
      for (int i = 0; i < (a.b0 < a.b1 ? a.pairs : 0) && ok; ++i) {
        ok = wait_warp(bar(st.k_full[rk.s]), rk.parity);
        for (int b = a.b0; b < a.b1 && ok; ++b) {
          const uint32_t cols = (block_cols(a, b, g) + 15) & ~15;
          const uint32_t idesc = idesc_bf16(kTileKeys, 0, false, false) | ((cols >> 3) << 17);
          if (i == 0) ok = wait_warp(bar(st.q_full[rq.s]), rq.parity);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            ok = ok && wait_warp(bar(st.s_empty[t][rs.s]), rs.parity ^ 1);
            if (!ok) break;
            tc_fence_after();
            mma_keys_e(st.tmem_base + t * 256 + rs.s * 128,
                       kdesc0 + (rk.s * kStageBytes + t * kBlockBytes) / 16, qdesc0 + rq.s * (kQBytes / 16), ones,
                       ldesc0 + rq.s * (kExtraBytes / 16), idesc,
                       bar(st.s_full[t][rs.s]));
          }
          if (!ok) break;
          if (i == a.pairs - 1) {  // a run of units keeps its block of queries
            tc_commit_e(bar(st.q_empty[rq.s]));
            rq.next();
          }
          rs.next();
        }
        if (!ok) break;
        tc_commit_e(bar(st.k_empty[rk.s]));
        rk.next();
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(bar(st.unit_empty[ru.s]));
      __syncwarp();
      ru.next();
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
    tc_commit_e(bar(st.drain));  // MMAs still in flight must not outlive TMEM
    mbar_wait(bar(st.drain), 0);
  } else if (warp == 2) {
    // ---------------------------------------------------------- earlier weights
    RingAt<kUnits> ru;
    RingAt<kOldStages> ro;
    bool ok = true;
    while (ok) {
      ok = wait_warp(bar(st.unit_full[ru.s]), ru.parity);
      if (!ok) break;
      const Unit a = st.units[ru.s];
      if (a.row < 0) break;
      const int old_end = a.slot < 0 && p.decay != 0.f ? a.len - a.n : 0;
      const float* w = p.weights + ((size_t)a.row * Hkv + a.kvh) * p.max_slots;
      for (int i = 0, k0 = a.k0; i < a.pairs; ++i, k0 += kUnitKeys) {
        ok = wait_warp(bar(st.old_empty[ro.s]), ro.parity ^ 1);
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < kUnitKeys / 32; ++k) {
          const int x = 32 * k + lane;
          if (k0 + x < old_end) copy_word(smem_addr(&st.old[ro.s][x]), w + k0 + x);
        }
        copies_arrive(bar(st.old_full[ro.s]));
        ro.next();
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(st.unit_empty[ru.s]));
      __syncwarp();
      ru.next();
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
    copies_wait();  // none in flight when the block ends
  } else if (warp >= 4 && warp < 4 + kQueryWarps) {
    // ---------------------------------------------------------------- queries
    // The warps take turns, a block each, so that as many are on their way.
    RingAt<kQStages> rq;
    RingAt<kUnits> ru;
    const int log_g = __ffs(g) - 1;
    uint32_t boxes = 0, turn = warp - 4;
    bool ok = true;
    while (ok) {
      ok = wait_warp(bar(st.unit_full[ru.s]), ru.parity);
      if (!ok) break;
      const Unit a = st.units[ru.s];
      if (a.row < 0) break;
      const int32_t* path = p.path ? p.path + (size_t)a.row * p.max_path : nullptr;
      for (int b = a.b0; b < a.b1; ++b, rq.next(), turn = turn == 0 ? kQueryWarps - 1 : turn - 1) {
        if (turn != 0) continue;
        const int cols = block_cols(a, b, g), t0 = b * (kCols >> log_g);
        const bool box = !path && cols == kCols;
        // (query token, q head) row of a column
        auto source = [&](int c) -> size_t {
          const int i = t0 + (c >> log_g);
          return (size_t)(a.q0 + (path ? path[i] : i)) * Hq + (a.kvh << log_g) + (c & (g - 1));
        };
        float nl[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          nl[k] = INFINITY;
          if (32 * k + lane < cols) nl[k] = p.lse[source(32 * k + lane)];
        }
        uint4 v[8];  // 32 columns' rows, four of them at a time
        auto load = [&](int c0) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int c = c0 + 4 * k + (lane >> 3);
            v[k] = make_uint4(0u, 0u, 0u, 0u);
            if (c < cols) v[k] = reinterpret_cast<const uint4*>(p.q + source(c) * kHeadDim)[lane & 7];
          }
        };
        if (!box) load(0);
        ok = wait_warp(bar(st.q_empty[rq.s]), rq.parity ^ 1);
        if (!ok) break;
        if (box) {
          if (lane == 0) {
            mbar_arrive_expect_tx(bar(st.q_full[rq.s]), kQBytes);
            tma_load_3d(sQ + rq.s * kQBytes, &qmap, 0, a.kvh << log_g, a.q0 + t0, bar(st.q_full[rq.s]));
          }
          __syncwarp();
        } else {
#pragma unroll 1
          for (int c0 = 0; c0 < cols; c0 += 32) {
            if (c0 > 0) load(c0);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const int c = c0 + 4 * k + (lane >> 3);
              *reinterpret_cast<uint4*>(base_ptr + (sQ - base) + rq.s * kQBytes + swz128(c, lane & 7)) = v[k];
            }
          }
          // The last query's once more in the columns that fill the product up, all
          // but weightless there: seen by the keys that see it, they add nothing that
          // it does not (zeros would: 0 * inf is NaN).
          const int spare = -cols & 15;
          if (spare) {
            uint8_t* stage = base_ptr + (sQ - base) + rq.s * kQBytes;
            __syncwarp();
#pragma unroll 1
            for (int i = lane; i < 8 * spare; i += 32) {
              const int c = cols + (i >> 3);
              *reinterpret_cast<uint4*>(stage + swz128(c, i & 7)) =
                  *reinterpret_cast<const uint4*>(stage + swz128(cols - g + (c & (g - 1)), i & 7));
            }
          }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          // an infinite lse, of a query that saw nothing too, leaves weights of 0
          const int c = 32 * k + lane;
          const float x = c >= cols ? -3e38f : nl[k] == -INFINITY ? -INFINITY : -nl[k] * p.inv_scale;
          const __nv_bfloat16 hi = __float2bfloat16_rn(x);
          const float r1 = x - __bfloat162float(hi);
          const __nv_bfloat16 mid = __float2bfloat16_rn(r1);
          const float r2 = r1 - __bfloat162float(mid);
          const bool inf = fabsf(x) == INFINITY;
          *reinterpret_cast<uint4*>(base_ptr + (sLse - base) + rq.s * kExtraBytes + 16 * c) =
              make_uint4((uint32_t)__bfloat16_as_ushort(hi) | (inf ? 0u : (uint32_t)__bfloat16_as_ushort(mid) << 16),
                         inf ? 0u : pack_bf16x2(r2, 0.f), 0u, 0u);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) {
          if (!box) mbar_arrive(bar(st.q_full[rq.s]));
          mbar_arrive(bar(st.q_full[rq.s]));
        }
        __syncwarp();
        if (box) boxes |= 1u << (2 * rq.s + rq.parity);  // stages and turns it has sent a box to
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(bar(st.unit_empty[ru.s]));
      __syncwarp();
      ru.next();
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
    // after an abort: wait (bounded) for boxes still in flight
    if (*abort_flag && lane == 0)
      for (uint32_t s = 0; s < 2 * kQStages; ++s)
        if (boxes >> s & 1u) mbar_wait(bar(st.q_full[s >> 1]), s & 1u);
  } else if (warp >= 8) {
    // ----------------------------------------------------------- exponentials
    // Two groups of eight warps take the blocks in turn, the second buffer of S
    // the second group's. Where a unit's blocks are one, the group that has it
    // finishes the unit; else the first group, with the second's sums.
    const int group = (warp - 8) >> 3, part = warp & 7, t = part >> 2;  // tile t
    const int key = part * 32 + lane;                                  // of the unit
    const uint32_t tmem_s = st.tmem_base + t * 256 + group * 128 + ((uint32_t)((warp & 3) * 32) << 16);
    const uint64_t sc = pack_f32x2(p.scale_log2, p.scale_log2);
    RingAt<kKStages> rk;
    RingAt<kOldStages> ro;
    RingAt<kUnits> ru;
    uint32_t cnt = 0, sums = 0;  // blocks, sums handed over
    const int W = p.window;
    bool ok = true;
    while (ok) {
      ok = wait_warp(bar(st.unit_full[ru.s]), ru.parity);
      if (!ok) break;
      const Unit a = st.units[ru.s];
      if (a.row < 0) break;
      const int C = a.len - a.n, blocks = a.b1 - a.b0;
      float* w = p.weights + ((size_t)a.row * Hkv + a.kvh) * p.max_slots;
      const int old_end = a.slot < 0 && p.decay != 0.f ? C : 0;
      int j = a.k0 + key;
      for (int i = 0; i < a.pairs; ++i, j += kUnitKeys) {
        const int first = j - lane;
        const bool busy = first < a.len;
        const bool finishes = blocks == 1 ? (int)(cnt & 1) == group : group == 0;
        uint32_t pages = 0;
        if (finishes && blocks > 0) {
          ok = wait_warp(bar(st.k_full[rk.s]), rk.parity);
          if (!ok) break;
          pages = st.pages[rk.s];
          __syncwarp();
          mbar_arrive_e(bar(st.k_empty[rk.s]));
        }
        if (blocks > 0) rk.next();
        float total = 0.f;
        for (int b = a.b0; b < a.b1; ++b, ++cnt) {
          if ((int)(cnt & 1) != group) continue;
          const int cols = (block_cols(a, b, g) + 15) & ~15, t0 = b * (kCols / g);
          ok = wait_warp(bar(st.s_full[t][group]), (cnt >> 1) & 1);
          if (!ok) break;
          tc_fence_after();
          uint64_t sum[2] = {0, 0};
          // hidden from some query of the block: keys behind its first, or before the window of its last
          const int tl = min(t0 + kCols / g, a.n) - 1;
          const bool plain = first + 31 <= C + t0 && (W == 0 || C + tl - first < W);
          if (busy) {
            const int lo = min(max(j - C - t0, 0), kCols) * g;
            const int hi = W == 0 ? kCols * kMaxGroup
                                  : (int)min(max((int64_t)j + W - C - t0, (int64_t)0), (int64_t)kCols) * g;
            uint32_t sv[32];
            if (plain && cols == kCols) {
#pragma unroll
              for (int c = 0; c < kCols; c += 32) {
                tmem_ld32(tmem_s + c, sv);
                tmem_ld_wait_for(sv);
                add_columns<32, false>(sv, sc, 0, 0, sum);
              }
            } else {
#pragma unroll 1
              for (int c = 0; c < cols; c += 32) {
                if (c + 32 <= cols) {
                  tmem_ld32(tmem_s + c, sv);
                  tmem_ld_wait_for(sv);
                  if (plain) add_columns<32, false>(sv, sc, 0, 0, sum);
                  else add_columns<32, true>(sv, sc, lo - c, hi - c, sum);
                } else {
                  tmem_ld16(tmem_s + c, sv);
                  tmem_ld_wait_for(sv);
                  if (plain) add_columns<16, false>(sv, sc, 0, 0, sum);
                  else add_columns<16, true>(sv, sc, lo - c, hi - c, sum);
                }
              }
            }
          }
          tc_fence_before();
          __syncwarp();
          mbar_arrive_e(bar(st.s_empty[t][group]));
          const uint64_t both = add2(sum[0], sum[1]);
          total += lo_f32(both) + hi_f32(both);
        }
        if (!ok) break;
        if (blocks > 1) {
          if (group == 1) {
            ok = wait_warp(bar(st.sum_empty[part]), (sums & 1) ^ 1);
            if (!ok) break;
            st.sums[key] = total;
            __syncwarp();
            mbar_arrive_e(bar(st.sum_full[part]));
          } else {
            ok = wait_warp(bar(st.sum_full[part]), sums & 1);
            if (!ok) break;
            total += st.sums[key];
            __syncwarp();
            mbar_arrive_e(bar(st.sum_empty[part]));
          }
          ++sums;
        }
        if (finishes) {
          ok = wait_warp(bar(st.old_full[ro.s]), ro.parity);
          if (!ok) break;
          const float old = j < old_end ? st.old[ro.s][key] : 0.f;
          __syncwarp();
          mbar_arrive_e(bar(st.old_empty[ro.s]));
          // a key that some query sees, on a page that is missing, keeps its weight
          const bool seen = j >= C || W == 0 || (int64_t)j + W > C;
          if (a.slot >= 0)
            p.parts[(size_t)a.slot * kUnitKeys + key] = total;
          else if (j < a.len && (!seen || (pages >> (key / kPage) & 1u)))
            w[j] = p.decay * old + total;
        }
        ro.next();
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(st.unit_empty[ru.s]));
      __syncwarp();
      ru.next();
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
  }
  __syncwarp();
  leave();
}

// The units that were cut: old weights and the parts, in the order of the
// pieces. Block c: the unit whose first part lies in piece c, if there is one.
__global__ void __launch_bounds__(kUnitKeys) merge_weights_kernel(const WeightParams p) {
  grid_dep_wait();
  const int4 cut = p.cuts[blockIdx.x];
  const int last = cut.x, r = cut.y, kvh = cut.z, j = cut.w + threadIdx.x;
  if (last < 0) return;
  const int S = p.seq_lens[r], n = p.path ? p.path_len[r] : p.qsl[r + 1] - p.qsl[r], C = S - n;
  if (j >= S) return;
  const int page = p.block_table[(size_t)r * p.max_pages + j / kPage];
  const bool seen = j >= C || p.window == 0 || (int64_t)j + p.window > C;
  if (seen && (page < 0 || page >= p.num_pages)) return;
  float* w = p.weights + ((size_t)r * p.num_kv_heads + kvh) * p.max_slots + j;
  float sum = p.parts[(size_t)(2 * blockIdx.x + 1) * kUnitKeys + threadIdx.x];
  for (int c = blockIdx.x + 1; c <= last; ++c) sum += p.parts[(size_t)(2 * c) * kUnitKeys + threadIdx.x];
  *w = (j < C && p.decay != 0.f ? p.decay * *w : 0.f) + sum;
}

}  // namespace

cudaError_t launch_weights(const CUtensorMap& kmap, const CUtensorMap& qmap, const WeightParams& p, int sms,
                           cudaStream_t stream) {
  const int grid = sms < kWeightCtas ? sms : kWeightCtas;
  LaunchCfg lc(dim3(grid), dim3(kThreads), weights_smem_bytes(), stream, true);
  const cudaError_t e = cudaLaunchKernelEx(&lc.cfg, weights_kernel, kmap, qmap, p);
  if (e != cudaSuccess) return e;
  // no row has more than kWholeBlocks blocks of queries: nothing is cut (a path
  // may name a query more than once, and more of them than the step has)
  const int64_t most = p.path ? p.max_path : p.total_q;
  if (most * p.group <= kWholeBlocks * kCols) return cudaSuccess;
  LaunchCfg mc(dim3(grid), dim3(kUnitKeys), 0, stream, true);
  return cudaLaunchKernelEx(&mc.cfg, merge_weights_kernel, p);
}

cudaError_t prepare_weights_kernels() {
  return cudaFuncSetAttribute(weights_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)weights_smem_bytes());
}

}  // namespace mcpu
