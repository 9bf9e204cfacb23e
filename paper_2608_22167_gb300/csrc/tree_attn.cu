// Paged attention of drafted-token trees (mcpu_tree_attention_forward) on the
// 5th-generation tensor cores (tcgen05 + TMEM).
//
// o_t = sum_{j in V(t)} e^{s_j - m} v_j / sum_{j in V(t)} e^{s_j - m},  s_j = scale q_t . k_j
// where V(t) holds the row's context keys (inside the window of t's position)
// and the nodes whose bit is set in t's mask.
//
// Work: a tile is 128 query rows of one (row, kv head): 128 / g nodes x the g
// heads; it walks the row's keys in blocks of 128 (8 pages). One CTA per SM
// runs two lanes, each a complete pipeline for one tile at a time (softmax,
// MMA issue, TMA, rings and barriers of its own), so that one lane's latencies
// are the other's work. The tiles are laid on two lines, each block weighing
// one and each tile kCostItem more:
//   solo   a row's last tile when their number is odd (all of a tree of up to
//          16 nodes at g = 8); cut into equal pieces, one per lane;
//   joint  the other tiles, in pairs that read the same keys; cut into equal
//          pieces, one per CTA, whose two lanes walk the pair side by side,
//          so that the second read of a K/V block finds it in L2.
// Whatever the lengths, every lane gets the same share. A tile that crosses a
// cut is computed in parts that merge_tree_kernel joins by log-sum-exp in the
// order of the pieces. Every CTA derives the lines from seq_lens and
// query_start_loc itself (prefix sums over the rows): no planning launch.
//
// Warps: 0, 1 issue S = Q K^T of lane 0, 1 (M 128, N 128, K 64) and 2, 3 issue
// O += P V (M 128, N 64, K 128, P from TMEM): an issuing warp is held until the
// tensor pipe takes its MMAs, and one warp for both had no time left in a block
// (2 % slower); 4, 5 bring K, the Q tiles, the parts and what the softmax
// needs of their masks, 6, 7 bring V (TMA, one 2 KiB box per page); 8-11 /
// 12-15 softmax of lane 0 / 1 (thread t owns row t & 127, a TMEM lane: running
// max and sum in fp32, P to TMEM as bf16 - each weight rounded once, 2^-8
// relative - and O rescaled only when the reference has to rise). The softmax
// takes 168 registers, the others give back all but 88. TMEM: per lane S 128,
// O 64, P 64 columns.
//
// Bound: reading K/V (2 KiB per key and 8 kv heads, once) up to 16 nodes at
// g = 8; from there the softmax, whose two warps per SM sub-partition take
// about 1650 cycles for a block of both lanes (1024 of exponentials at 8 a
// clock; the same instructions without waits 1330, with barriers that are
// always ready 1460). Its loop over plain blocks is kept apart from all that is
// rare: with masks, first blocks and rescaling inside it, it took 2430, much of
// it waiting for instructions. Measured on a GB300: 64 rows of 2k-16k keys with
// 1-16 nodes 192-195 us (6.3 TB/s of K/V), 4k-32k keys with 16-32 nodes 533-566
// us (805-860 TFLOP/s, by the clock that the power limit leaves), two rows of
// 49k-65k keys with 61 and 64 nodes 114-117 us (1010-1030 TFLOP/s), 384 rows in
// a window of 128 keys 94 us, four rows of up to 308 keys 9.3 us (11.7 where a
// wide table has the merge launched).
//
// Waits are bounded; one that runs out raises an abort flag, every role ends,
// and TMEM is freed after the issuers' MMAs have drained.
//
// What the caller gives is read by ordinary loads (not the non-coherent ones):
// the grid may be placed while the one that writes it still runs.
#include "tcgen05.cuh"
#include "tree_round.cuh"
#include "warp_pipe.cuh"

namespace mcpu {

namespace {

constexpr int kTileRows = kTreeTileRows;  // query rows of one tile (TMEM lanes)
constexpr int kKStages = 3, kVStages = 2;            // per lane
constexpr int kQBytes = kTileRows * kRowBytes;
constexpr int kLaneBytes = kQBytes + (kKStages + kVStages) * kBlockBytes;
constexpr int kTreeThreads = 512;
constexpr int kHelperRegs = 88, kSoftmaxRegs = 168;  // of 128 at launch: two warpgroups each
static_assert(2 * (kHelperRegs + kSoftmaxRegs) == 4 * 128, "the registers of the launch");
constexpr uint32_t kTmemCols = 512;
constexpr int kCostItem = 5;  // a tile's set-up and end, in blocks
constexpr int kWholeBlocks = 6;  // tiles of up to so many blocks are never cut
constexpr int kMinQuota = 7;  // smallest piece worth a lane of its own

struct alignas(16) Part {  // a run of key blocks of one tile
  int32_t row;                 // -1: no more parts
  int32_t token, n_tok, node;  // first query token, tokens, first node of the tile
  int32_t ctx, len, kvh;
  int32_t kb0;  // key of block 0 (a page start)
  int32_t b0, b1;
  int32_t slot;  // partial slot, or -1: the part is the whole tile
};

struct Meta {  // what the softmax needs to know of a part's nodes
  uint32_t seen_by_any[MCPU_MAX_TREE_WORDS];  // nodes that some node of the row sees
  int32_t first;                              // first context key that some node of the row sees
  float sinks[kMaxGroup];                     // base-2 sink logits of the kv head's query heads
  int32_t lo[kTileRows];                      // first context key in each node's window
  uint32_t mask[kTileRows * MCPU_MAX_TREE_WORDS];  // [node of the tile][words]
};

struct Lane {
  uint64_t q_full, q_empty;
  uint64_t k_full[kKStages], k_empty[kKStages], v_full[kVStages], v_empty[kVStages];
  uint64_t s_full, s_free, p_full, o_ready, o_free;
  uint64_t part_full[2], part_empty[2], meta_full[2];
  uint64_t drain[2];
  Part parts[2];
  Meta meta[2];
};

struct TreeSmem {
  Lane lane[2];
  int64_t scan[2][kTreeThreads / 32];
  int64_t first_off[3];  // where a piece begins in its first row: solo of lane 0, of lane 1, joint
  int32_t first_row[3];
  uint32_t tmem_base;
  int32_t abort_flag;
};

static_assert(2 * kLaneBytes >= 2 * (kMaxSeqs + 1) * (int)sizeof(int64_t), "the prefix sums use the rings first");

size_t tree_smem_bytes() { return 1024 + 2 * (size_t)kLaneBytes + sizeof(TreeSmem); }

// ----------------------------------------------------------- the work lines
struct RowGeom {
  int q0, L, S, C, key_begin, kb0, nb;
  int pairs, solo;  // joint pairs of tiles, and 1 if a last tile stands alone
  __device__ int64_t cost() const { return kCostItem + nb; }  // of one tile
};

// Geometry of row r; false (L = 0: nothing wrong) if it has no work, with the
// status bits of what is wrong.
__device__ __forceinline__ bool row_geom(const TreeParams& p, int r, RowGeom* w, int32_t* bits) {
  w->q0 = p.qsl[r];
  w->L = p.qsl[r + 1] - w->q0;
  w->S = p.seq_lens[r];
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
  const int tiles = (w->L * p.group + kTileRows - 1) / kTileRows;
  w->pairs = tiles >> 1;
  w->solo = tiles & 1;
  return true;
}

// Blocks of a tile of nb blocks that belong to the pieces ending x units into
// it. A short tile is not cut (its parts would each pay for a set-up, and for
// the merge): all of it belongs to the piece it begins in.
__device__ __forceinline__ int blocks_before(int64_t x, int nb) {
  if (nb <= kWholeBlocks) return x <= 0 ? 0 : nb;
  return x <= kCostItem ? 0 : x >= kCostItem + nb ? nb : (int)(x - kCostItem);
}

// ceil(a / b), a + b > 0; the 64-bit division, which is long, in one place.
__device__ __noinline__ int64_t div_long(int64_t a, int64_t b) { return a / b; }
__device__ __forceinline__ int64_t div_up(int64_t a, int32_t b) {
  const int64_t n = a + b - 1;
  return n >> 32 ? div_long(n, b) : (int64_t)((uint32_t)n / (uint32_t)b);
}

// Whether a part names rows of this call: what is read from shared memory
// becomes addresses, so every role checks it before it uses it.
__device__ __forceinline__ bool part_ok(const TreeParams& p, const Part& a) {
  return a.row < p.num_seqs && a.token >= 0 && a.n_tok >= 1 && a.n_tok * p.group <= kTileRows &&
         a.token <= p.total_q - a.n_tok && a.kvh >= 0 && a.kvh < p.num_kv_heads && a.b0 >= 0 && a.b1 > a.b0 &&
         a.slot >= -1 && a.slot < kTreeSlots && a.ctx >= 0 && a.len <= p.max_pages * kPage && a.node >= 0 &&
         a.node + a.n_tok <= a.len - a.ctx && a.len - a.ctx <= 32 * p.words;
}

// The MMAs of S and of O with the commits behind them, issued by one elected
// lane of a warp in step.
__device__ __forceinline__ void mma_scores_e(uint32_t d, uint64_t q, uint64_t k, uint32_t idesc, uint32_t done,
                                             uint32_t k_free) {
  static_assert(kHeadDim == 64, "four steps of 16 dims, 32 bytes each");
  asm volatile(
      "{\n\t.reg .pred e, t, f;\n\t.reg .b64 a, b;\n\telect.sync _|e, 0xffffffff;\n\t"
      "setp.eq.u32 t, 0, 0;\n\tsetp.ne.u32 f, 0, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, f;\n\t"
      "add.s64 a, %1, 2;\n\tadd.s64 b, %2, 2;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
      "add.s64 a, %1, 4;\n\tadd.s64 b, %2, 4;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
      "add.s64 a, %1, 6;\n\tadd.s64 b, %2, 6;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, t;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%4];\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t"
      "}" ::"r"(d),
      "l"(q), "l"(k), "r"(idesc), "r"(done), "r"(k_free)
      : "memory");
}
__device__ __forceinline__ void mma_values_e(uint32_t d, uint32_t pw, uint64_t v, uint32_t idesc, uint32_t add,
                                             uint32_t done, uint32_t v_free) {
  static_assert(kBlockKeys == 128 && 16 * kRowBytes / 16 == 128, "eight steps of 16 keys, 2 KiB of V each");
  asm volatile(
      "{\n\t.reg .pred e, t, f;\n\t.reg .b32 a;\n\t.reg .b64 b;\n\telect.sync _|e, 0xffffffff;\n\t"
      "setp.eq.u32 t, 0, 0;\n\tsetp.ne.u32 f, %4, 0;\n\t"
      "@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, f;\n\t"
      "add.s32 a, %1, 8;\n\tadd.s64 b, %2, 128;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "add.s32 a, %1, 16;\n\tadd.s64 b, %2, 256;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "add.s32 a, %1, 24;\n\tadd.s64 b, %2, 384;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "add.s32 a, %1, 32;\n\tadd.s64 b, %2, 512;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "add.s32 a, %1, 40;\n\tadd.s64 b, %2, 640;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "add.s32 a, %1, 48;\n\tadd.s64 b, %2, 768;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "add.s32 a, %1, 56;\n\tadd.s64 b, %2, 896;\n\t@e tcgen05.mma.cta_group::1.kind::f16 [%0], [a], b, %3, t;\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%5];\n\t"
      "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%6];\n\t"
      "}" ::"r"(d),
      "r"(pw), "l"(v), "r"(idesc), "r"(add), "r"(done), "r"(v_free)
      : "memory");
}

// ------------------------------------------------------------------ softmax
// the low n bits (none for n <= 0, all for n >= 32)
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }

__device__ __forceinline__ void hide(uint32_t (&sv)[32], uint32_t seen) {
  if (!__any_sync(0xffffffffu, seen != 0xffffffffu)) return;  // most words of a masked block are plain context
#pragma unroll
  for (int e = 0; e < 32; ++e)
    if (!(seen >> e & 1u)) sv[e] = 0xff800000u;
}

// pk[at ..] = bf16(2^(s * scale - mu)) of 32 scores; their fp32 sum (before
// rounding) goes to sum.
template <int at>
__device__ __forceinline__ void weights(const uint32_t (&sv)[32], uint64_t sc, uint64_t mu, uint64_t (&sum)[2],
                                        uint32_t (&pk)[32]) {
#pragma unroll
  for (int e = 0; e < 32; e += 2) {
    const uint64_t x = fma2((uint64_t)sv[e] | ((uint64_t)sv[e + 1] << 32), sc, mu);
    const float p0 = ex2_approx(lo_f32(x)), p1 = ex2_approx(hi_f32(x));
    sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pack_f32x2(p0, p1));
    pk[at + e / 2] = pack_bf16x2(p0, p1);
  }
}
__device__ __forceinline__ float sum_of(const uint64_t (&sum)[2]) {
  const uint64_t s = add2(sum[0], sum[1]);
  return lo_f32(s) + hi_f32(s);
}

__device__ __forceinline__ float scores_max(const uint32_t (&sv)[32]) {
  float m[2] = {-INFINITY, -INFINITY};
#pragma unroll
  for (int e = 0; e < 32; e += 4)
#pragma unroll
    for (int k = 0; k < 2; ++k)
      m[k] = fmax3(m[k], __uint_as_float(sv[e + 2 * k]), __uint_as_float(sv[e + 2 * k + 1]));
  return fmaxf(m[0], m[1]);
}

template <int at>
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[32]) {  // 16 TMEM columns from v[at ..]
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16};" ::"r"(taddr),
      "r"(v[at]), "r"(v[at + 1]), "r"(v[at + 2]), "r"(v[at + 3]), "r"(v[at + 4]), "r"(v[at + 5]), "r"(v[at + 6]),
      "r"(v[at + 7]), "r"(v[at + 8]), "r"(v[at + 9]), "r"(v[at + 10]), "r"(v[at + 11]), "r"(v[at + 12]),
      "r"(v[at + 13]), "r"(v[at + 14]), "r"(v[at + 15])
      : "memory");
}

__device__ __forceinline__ void zero_smem16(uint32_t addr) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(addr), "r"(0u) : "memory");
}

// Which of the keys k0 .. k0 + 31 the thread's node (of the tile) sees.
__device__ __forceinline__ uint32_t seen_keys(const TreeParams& p, const Part& a, const Meta& m, int node, int k0) {
  const int lo = p.window > 0 ? m.lo[node] : 0, n0 = k0 - a.ctx;
  uint32_t seen = low_bits(-n0) & ~low_bits(lo - k0);
  if (n0 > -32) {  // the nodes n0 .. are bits of two mask words
    const uint32_t* w = m.mask + node * p.words;
    const int i = n0 >> 5;
    const uint32_t first = i >= 0 && i < p.words ? w[i] : 0u, second = i + 1 < p.words ? w[i + 1] : 0u;
    seen |= __funnelshift_r(first, second, n0 & 31) & low_bits(a.len - k0);
  }
  return seen;
}

// Whether slot j holds a V row that no node of the row sees.
__device__ __forceinline__ bool dead_slot(const Part& a, const Meta& m, int j) {
  const int n = j - a.ctx;
  if (n < 0) return j < m.first;
  // past the row's end only its last page holds anything: later pages arrive as zeros
  if (j >= a.len) return j < ((a.len + kPage - 1) & ~(kPage - 1));
  return !(m.seen_by_any[n >> 5] >> (n & 31) & 1u);
}

__device__ __forceinline__ float tree_sink(const TreeParams& p, int h) {
  return p.sinks ? p.sinks[h] * 1.4426950408889634f : -INFINITY;
}

// --------------------------------------------------------------- the kernel
__global__ void __launch_bounds__(kTreeThreads, 1)
    tree_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                const __grid_constant__ CUtensorMap qmap, const TreeParams p) {
  extern __shared__ uint8_t smem_raw[];
  // (through lane 0, so that what follows from the warp's role is known to be uniform)
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const uint32_t raw = smem_addr(smem_raw);
  const uint32_t base = (raw + 1023u) & ~1023u;
  uint8_t* base_ptr = smem_raw + (base - raw);
  TreeSmem& st = *reinterpret_cast<TreeSmem*>(base_ptr + 2 * kLaneBytes);
  int64_t* prefix = reinterpret_cast<int64_t*>(base_ptr);  // [2][B + 1], until the parts begin
  volatile int32_t* abort_flag = &st.abort_flag;
  auto bar = [&](uint64_t& b) { return smem_addr(&b); };
  const int B = p.num_seqs, g = p.group, Hkv = p.num_kv_heads, Hq = p.num_q_heads;

  // Before anything is read: TMEM, the barriers, the tensor maps.
  if (warp == 0) {
    tmem_alloc(smem_addr(&st.tmem_base), kTmemCols);
    tmem_relinquish();
  }
  if (threadIdx.x >= 32 && threadIdx.x < 34) {
    Lane& ln = st.lane[threadIdx.x - 32];
    mbar_init(bar(ln.q_full), 1);
    mbar_init(bar(ln.q_empty), 1);
    for (int s = 0; s < kKStages; ++s) {
      mbar_init(bar(ln.k_full[s]), 1);
      mbar_init(bar(ln.k_empty[s]), 1);
    }
    for (int s = 0; s < kVStages; ++s) {
      mbar_init(bar(ln.v_full[s]), 1);
      mbar_init(bar(ln.v_empty[s]), 1);
    }
    mbar_init(bar(ln.s_full), 1);
    mbar_init(bar(ln.s_free), 4);
    mbar_init(bar(ln.p_full), 4);
    mbar_init(bar(ln.o_ready), 1);
    mbar_init(bar(ln.o_free), 4);
    for (int i = 0; i < 2; ++i) {
      mbar_init(bar(ln.part_full[i]), 1);
      mbar_init(bar(ln.part_empty[i]), 4 + 2);
      mbar_init(bar(ln.meta_full[i]), 1);
    }
    mbar_init(bar(ln.drain[0]), 1);
    mbar_init(bar(ln.drain[1]), 1);
    st.abort_flag = 0;
    fence_barrier_init();
  }
  if (threadIdx.x == 64) {
    prefetch_tensormap(&kmap);
    prefetch_tensormap(&vmap);
    prefetch_tensormap(&qmap);
  }
  auto leave = [&] {  // the whole CTA
    tc_fence_before();
    __syncthreads();
    if (warp == 0) {
      tc_fence_after();
      tmem_dealloc(st.tmem_base, kTmemCols);
    }
  };

  // The merge may be launched from now on (its blocks find no room until this
  // grid's CTAs leave, and wait for its end); nothing is read before the grid
  // that this one follows has ended.
  grid_dep_launch();
  grid_dep_wait();
  // no cut tile begins in this CTA's pieces, as far as is known
  if (threadIdx.x < 4)
    p.cuts[(threadIdx.x >> 1) * 2 * gridDim.x + 2 * blockIdx.x + (threadIdx.x & 1)] = make_int4(-1, 0, 0, 0);
  const bool ends = p.qsl[0] == 0 && p.qsl[B] == p.total_q;
  // ---- the lines: prefix[l][r] = cost of line l's tiles in the rows before r
  {
    const int per = (B + kTreeThreads - 1) / kTreeThreads;
    const int r0 = min(B, (int)threadIdx.x * per), r1 = min(B, r0 + per);
    int64_t sum[2] = {0, 0};
    int32_t bits = 0;
    RowGeom w;
    int64_t tail[2] = {0, 0};  // the last row's
    for (int r = r0; r < r1; ++r) {
      const bool any = row_geom(p, r, &w, &bits);
      tail[0] = any ? w.cost() * Hkv * w.solo : 0;
      tail[1] = any ? w.cost() * Hkv * w.pairs : 0;
      sum[0] += tail[0];
      sum[1] += tail[1];
    }
    if (!ends) bits = threadIdx.x == 0 ? kStatusBadLengths : 0;
    if (bits && blockIdx.x == 0) atomicOr(p.status, bits);
    int64_t at[2];
#pragma unroll
    for (int l = 0; l < 2; ++l) {
      int64_t incl = sum[l];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, (long long)incl, o);
        if (lane >= o) incl += v;
      }
      if (lane == 31) st.scan[l][warp] = incl;
      at[l] = incl - sum[l];
    }
    __syncthreads();
    for (int i = 0; i < warp; ++i) {
      at[0] += st.scan[0][i];
      at[1] += st.scan[1][i];
    }
    for (int r = r0; r < r1; ++r) {
      prefix[r] = at[0];
      prefix[B + 1 + r] = at[1];
      if (r + 1 == r1) {
        at[0] += tail[0];
        at[1] += tail[1];
      } else if (row_geom(p, r, &w, &bits)) {
        at[0] += w.cost() * Hkv * w.solo;
        at[1] += w.cost() * Hkv * w.pairs;
      }
    }
    if (threadIdx.x == kTreeThreads - 1) {
      prefix[B] = at[0];
      prefix[2 * B + 1] = at[1];
    }
  }
  __syncthreads();
  // pieces: solo of this CTA's lanes, then joint
  const int64_t total0 = prefix[B], total1 = prefix[2 * B + 1];
  const int64_t quota0 = max(div_up(total0, 2 * gridDim.x), (int64_t)kMinQuota);
  const int64_t quota1 = max(div_up(total1, gridDim.x), (int64_t)kMinQuota);
  const int64_t begin0 = 2 * (int64_t)blockIdx.x * quota0, begin1 = (int64_t)blockIdx.x * quota1;
  if (!ends || (begin0 >= total0 && begin1 >= total1)) return leave();  // uniform over the CTA
  if (warp < 3) {  // the row each piece begins in: warp 0, 1 solo of their lane, 2 joint
    const int l = warp == 2;
    const int64_t u = l ? begin1 : begin0 + warp * quota0;
    const int64_t* pre = prefix + l * (B + 1);
    int r0 = 0;
    for (int r = 1 + lane; r < B; r += 32) r0 += pre[r] <= u;  // pre[r0] <= u < pre[r0 + 1] if u is on the line
    r0 = __reduce_add_sync(0xffffffffu, r0);
    if (lane == 0) {
      st.first_row[warp] = r0;
      st.first_off[warp] = u - pre[r0];
    }
  }
  fence_proxy_async();  // the rings' first TMA writes come after the reads of the prefix sums
  tc_fence_before();
  __syncthreads();
  tc_fence_after();

  const int x = warp >= 8 ? (warp >> 2) - 2 : warp & 1;  // this warp's lane of the CTA
  Lane& ln = st.lane[x];
  const uint32_t sQ = base + x * kLaneBytes, sK = sQ + kQBytes, sV = sK + kKStages * kBlockBytes;
  const uint32_t tmem = st.tmem_base + x * 256;  // S at 0, O at 128, P at 192
  constexpr uint32_t kColO = 128, kColP = 192;

  // Each role is one or two whole warpgroups; the softmax takes the registers
  // that the others give back.
  if (warp >= 4 && warp < 8) {
    // ------------------------------------------------------------- producer
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHelperRegs));
    const bool for_k = warp < 6;  // K, Q tiles and the parts; else V
    RingAt<kKStages> rk;
    RingAt<kVStages> rv;
    uint32_t it = 0;  // blocks issued
    int i = 0;
    bool ok = true;
#pragma unroll 1
    for (int line = 0; line < 2 && ok; ++line) {
      const int64_t quota = line ? quota1 : quota0;
      const int64_t u0 = line ? begin1 : begin0 + x * quota0, u1 = min(u0 + quota, line ? total1 : total0);
      if (u0 >= u1) continue;
      const int which = line ? 2 : x;
      int row = st.first_row[which];
      RowGeom w;
      int32_t ignored = 0;
      row_geom(p, row, &w, &ignored);
      int64_t off = st.first_off[which];
      int item = 0;  // (kv head, pair) of the row
      for (; off >= w.cost(); off -= w.cost()) ++item;
      int64_t u = u0 - off;  // start of the current tile on the line
      // K/V of joint tiles is read by both lanes, of solo ones once
      const uint64_t pol = line ? policy_evict_last() : policy_evict_first();
      while (u < u1) {
        const int per_head = line ? w.pairs : 1, tile_tok = kTileRows / g;
        Part a;
        a.b0 = blocks_before(u0 - u, w.nb);
        a.b1 = blocks_before(u1 - u, w.nb);
        a.row = row;
        a.kvh = item / per_head;
        const int tile = line ? 2 * (item % per_head) + x : 2 * w.pairs;
        a.node = tile * tile_tok;
        a.token = w.q0 + a.node;
        a.n_tok = min(tile_tok, w.L - a.node);
        a.ctx = w.C;
        a.len = w.S;
        a.kb0 = w.kb0;
        const int first = a.b0 == 0 ? 1 : 0;
        a.slot = first && a.b1 == w.nb ? -1
                 : line                ? kTreeSoloSlots + (2 * (int)blockIdx.x + first) * 2 + x
                                       : 2 * (2 * (int)blockIdx.x + x) + first;
        if (first && a.slot >= 0 && a.b1 > 0 && for_k && lane == 0) {
          // a cut tile whose first part is this one: its last piece and what the merge needs
          int last = line ? blockIdx.x : 2 * blockIdx.x + x;
          for (int64_t end = u0 + quota; end < u + w.cost(); end += quota) ++last;
          p.cuts[line * 2 * gridDim.x + 2 * blockIdx.x + x] = make_int4(last, a.token, a.n_tok, a.kvh);
        }
        u += w.cost();
        if (++item == Hkv * per_head) {
          item = 0;
          do ++row;
          while (row < B && !(row_geom(p, row, &w, &ignored) && (line ? w.pairs : w.solo) > 0));
        }
        if (a.b0 >= a.b1) continue;
        const int slot = i & 1;
        if (!part_ok(p, a)) {
          atomicOr(p.status, kStatusPlanOverflow);
          *abort_flag = 2;
          ok = false;
          break;
        }
        // page ids and mask words are on their way while the slot empties
        const int* bt_row = p.block_table + (size_t)a.row * p.max_pages;
        const int n = a.b1 - a.b0, pg0 = a.kb0 / kPage + a.b0 * kBlockPages;
        const int page_end = min((a.len + kPage - 1) / kPage, pg0 + n * kBlockPages);
        auto load_ids = [&](int c) -> int {  // page id of page pg0 + 32c + lane
          const int lp = pg0 + 32 * c + lane;
          return lp < page_end ? bt_row[lp] : -2;
        };
        const int L = a.len - a.ctx;
        const int32_t* row_pos = p.positions + (a.token - a.node);  // with a window only
        auto first_key = [&](int pos) { return min(max(pos, a.ctx), a.len - 1) - p.window + 1; };
        // where the page's box begins; nothing past the last page, nor for a missing page that no node sees (nodes
        // may all lie past C, where the first block begins)
        auto box_row = [&](int id, int lp) -> int {
          if (id >= 0 && id < p.num_pages) return (id * Hkv + a.kvh) * kPage;
          bool seen = id != -2;
          if (seen && p.window > 0) {
            seen = false;
#pragma unroll 1
            for (int k = 0; k < L && !seen; ++k) seen = lp * kPage + kPage > min(first_key(row_pos[k]), a.ctx);
          }
          if (seen) atomicOr(p.status, kStatusBadPage);
          return p.oob_row;
        };
        int ids_next = load_ids(0);
        uint32_t early = 0;
        int early_pos = 0, early_row_pos = 0;
        float sink = -INFINITY;
        const uint32_t* rows = p.mask + (size_t)a.token * p.words;
        const int mine = a.n_tok * p.words;
        if (for_k) {
          if (lane < mine) early = rows[lane];
          if (p.window > 0 && lane < a.n_tok) early_pos = row_pos[a.node + lane];
          if (p.window > 0 && lane < L) early_row_pos = row_pos[lane];
          if (lane < g) sink = tree_sink(p, a.kvh * g + lane);
          ok = i < 2 || wait_warp(bar(ln.part_empty[slot]), ((i >> 1) - 1) & 1);
          if (!ok) break;
          if (lane == 0) {
            ln.parts[slot] = a;
            mbar_arrive(bar(ln.part_full[slot]));
          }
          __syncwarp();
          ok = i < 1 || wait_warp(bar(ln.q_empty), (i - 1) & 1);
          if (!ok) break;
          if (lane == 0) {
            mbar_arrive_expect_tx(bar(ln.q_full), kQBytes);
            tma_load_3d(sQ, &qmap, 0, a.kvh * g, a.token, bar(ln.q_full));
          }
          __syncwarp();
        }
        ++i;
        int at = 0;
#pragma unroll 1
        for (int b = 0; b < n; ++b) {
          if (!(b & 3)) {  // 32 pages: a lane each, the next ones' ids on their way
            at = box_row(ids_next, pg0 + kBlockPages * b + lane);
            ids_next = load_ids((b >> 2) + 1);
          }
          int y[kBlockPages];
#pragma unroll
          for (int j = 0; j < kBlockPages; ++j) y[j] = __shfl_sync(0xffffffffu, at, (b & 3) * kBlockPages + j);
          if (!for_k) {
            ok = wait_warp(bar(ln.v_empty[rv.s]), rv.parity ^ 1);
            if (!ok) break;
            load_block_e(sV + rv.s * kBlockBytes, &vmap, y, bar(ln.v_full[rv.s]), pol);
            rv.next();
            ++it;
            continue;
          }
          ok = wait_warp(bar(ln.k_empty[rk.s]), rk.parity ^ 1);
          if (!ok) break;
          load_block_e(sK + rk.s * kBlockBytes, &kmap, y, bar(ln.k_full[rk.s]), pol);
          rk.next();
          ++it;
          if (b > 0) continue;
          // behind the first K block: what the softmax needs of the masks
          Meta& m = ln.meta[slot];
          const uint32_t* all = rows - (size_t)a.node * p.words;
#pragma unroll 1
          for (int k = lane; k < mine; k += 32) m.mask[k] = k < 32 ? early : rows[k];
          int first = 0;
          if (p.window > 0) {
#pragma unroll 1
            for (int k = lane; k < a.n_tok; k += 32) m.lo[k] = first_key(k < 32 ? early_pos : row_pos[a.node + k]);
            first = a.ctx;
#pragma unroll 1
            for (int k = lane; k < L; k += 32) first = min(first, first_key(k < 32 ? early_row_pos : row_pos[k]));
            first = __reduce_min_sync(0xffffffffu, first);
          }
          if (lane == 0) m.first = first;
          if (a.b1 * kBlockKeys + a.kb0 > a.ctx)  // the part reaches the nodes
#pragma unroll 1
            for (int c = 0; c < p.words; ++c) {
              uint32_t any = 0;
#pragma unroll 1
              for (int k = lane; k < L; k += 32) any |= all[(size_t)k * p.words + c];
              any = __reduce_or_sync(0xffffffffu, any);
              if (lane == 0) m.seen_by_any[c] = any;
            }
          if (lane < g) m.sinks[lane] = sink;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(ln.meta_full[slot]));
          __syncwarp();
        }
        if (!ok) break;
      }
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
    if (ok && for_k && (i < 2 || wait_warp(bar(ln.part_empty[i & 1]), ((i >> 1) - 1) & 1))) {
      if (lane == 0) {  // no more parts
        ln.parts[i & 1].row = -1;
        mbar_arrive(bar(ln.part_full[i & 1]));
      }
    }
    // after an abort: wait (bounded) for the copies still in flight
    if (*abort_flag && lane == 0) {
      const uint32_t stages = for_k ? kKStages : kVStages;
      for (uint32_t k = it > stages ? it - stages : 0; k < it; ++k)
        mbar_wait(bar(for_k ? ln.k_full[k % stages] : ln.v_full[k % stages]), (k / stages) & 1);
      if (for_k && i > 0) mbar_wait(bar(ln.q_full), (i - 1) & 1);
    }
  } else if (warp < 4) {
    // -------------------------------------------- MMA issue: S, or O, of a lane
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kHelperRegs));
    constexpr uint32_t idS = idesc_bf16(kTileRows, kBlockKeys, false, false);
    constexpr uint32_t idO = idesc_bf16(kTileRows, kHeadDim, false, true);
    constexpr uint64_t kStageStep = kBlockBytes / 16;
    const bool for_s = warp < 2;
    const uint64_t kdesc0 = smem_desc_sw128(sK, 16, 1024), vdesc0 = smem_desc_sw128(sV, 1024, 1024);
    const uint64_t qd = smem_desc_sw128(sQ, 16, 1024);
    RingAt<kKStages> rk;
    RingAt<kVStages> rv;
    uint32_t par = for_s ? 1 : 0;  // turn of s_free, or of p_full
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int slot = i & 1;
      ok = wait_warp(bar(ln.part_full[slot]), (i >> 1) & 1);
      if (!ok || ln.parts[slot].row < 0) break;
      const int n = ln.parts[slot].b1 - ln.parts[slot].b0;
      if (for_s) {
        ok = wait_warp(bar(ln.q_full), i & 1);
        for (int b = 0; b < n && ok; ++b) {
          ok = wait_warp(bar(ln.k_full[rk.s]), rk.parity) && wait_warp(bar(ln.s_free), par);
          if (!ok) break;
          tc_fence_after();
          mma_scores_e(tmem, qd, kdesc0 + rk.s * kStageStep, idS, bar(ln.s_full), bar(ln.k_empty[rk.s]));
          if (b == n - 1) tc_commit_e(bar(ln.q_empty));
          rk.next();
          par ^= 1;
        }
      } else {
        ok = i == 0 || wait_warp(bar(ln.o_free), (i - 1) & 1);
        for (int b = 0; b < n && ok; ++b) {
          ok = wait_warp(bar(ln.v_full[rv.s]), rv.parity) && wait_warp(bar(ln.p_full), par);
          if (!ok) break;
          tc_fence_after();
          mma_values_e(tmem + kColO, tmem + kColP, vdesc0 + rv.s * kStageStep, idO, b > 0 ? 1u : 0u, bar(ln.o_ready),
                       bar(ln.v_empty[rv.s]));
          rv.next();
          par ^= 1;
        }
      }
      if (!ok) break;
      if (lane == 0) mbar_arrive(bar(ln.part_empty[slot]));
      __syncwarp();
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
    // MMAs still in flight (after an abort) must not outlive TMEM
    tc_commit_e(bar(ln.drain[for_s]));
    mbar_wait(bar(ln.drain[for_s]), 0);
  } else {
    // -------------------------------------------------------------- softmax
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int wq = warp & 3, row = threadIdx.x & (kTileRows - 1);
    const uint32_t cS = tmem + ((uint32_t)(wq * 32) << 16), cO = cS + kColO, cP = cS + kColP;
    const int tok = row / g, head = row % g;
    uint32_t cnt = 0;  // blocks so far: phase of every block barrier
    bool ok = true;
    for (int i = 0; ok; ++i) {
      const int slot = i & 1;
      ok = wait_warp(bar(ln.part_full[slot]), (i >> 1) & 1);
      if (!ok) break;
      const Part a = ln.parts[slot];
      if (a.row < 0) break;
      if (!part_ok(p, a)) {
        atomicOr(p.status, kStatusPlanOverflow);
        *abort_flag = 2;
        break;
      }
      ok = wait_warp(bar(ln.meta_full[slot]), (i >> 1) & 1);
      if (!ok) break;
      const int n = a.b1 - a.b0;
      const int my_node = min(tok, a.n_tok - 1);
      // blocks that need no mask: keys [plain_lo, ctx) are seen by every node
      const int plain_lo = p.window > 0 ? a.len - p.window : 0, plain_hi = a.ctx - kBlockKeys;
      int kb = a.kb0 + a.b0 * kBlockKeys;
      float m_ref = -INFINITY, l = 0.f;
      const bool busy = wq * 32 < a.n_tok * g;  // this warp has rows
      // V rows that no node sees may hold anything, and a zero weight does not
      // cancel a NaN: they are cleared before the PV reads them
      auto clear_dead = [&](bool dead) -> bool {
        if (!__any_sync(0xffffffffu, dead)) return true;
        const uint32_t s = cnt % kVStages;
        if (!wait_warp(bar(ln.v_full[s]), (cnt / kVStages) & 1)) return false;
        if (dead) {
#pragma unroll
          for (int c = 0; c < 8; ++c) zero_smem16(sV + s * kBlockBytes + row * kRowBytes + c * 16);
        }
        fence_proxy_async();
        return true;
      };
      if (!busy) {  // none of this warp's rows is a query: it only keeps the barriers and clears V rows
        for (int b = 0; b < n; ++b, ++cnt, kb += kBlockKeys) {
          const bool dead = (kb > plain_hi || kb < plain_lo) && dead_slot(a, ln.meta[slot], kb + row);
          ok = wait_warp(bar(ln.s_full), cnt & 1);
          if (!ok) break;
          if (lane == 0) mbar_arrive(bar(ln.s_free));
          // in step with the other warps: one arrival per phase
          if (cnt >= 1) {
            ok = wait_warp(bar(ln.o_ready), (cnt - 1) & 1);
            if (!ok) break;
          }
          ok = clear_dead(dead);
          if (!ok) break;
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(ln.p_full));
        }
      } else {
        bool unset = true;  // some row has no reference yet
        for (int b = 0; b < n; ++b, ++cnt, kb += kBlockKeys) {
          // ---- blocks that every node sees, all references set: a loop of its
          // own, small enough to stay in the instruction cache. Four chunks of
          // 32 scores, the next one's load in flight while one's weights are
          // made. Nothing is known of the scores before: weights up to 2^60 of
          // the first half are taken as they are (their row's sum shows it; else
          // the block is done anew below), and what exceeds 2^8 is scaled down
          // after the last. S is free for the next block's product before the
          // second half's weights are made.
          if (!unset) {
            const int stop = min(n, b + (min(plain_hi, a.kb0 + (a.b1 - 1) * kBlockKeys) - kb) / kBlockKeys + 1);
            const uint64_t sc = pack_f32x2(p.scale_log2, p.scale_log2);
            if (kb < plain_lo || kb > plain_hi) goto general;
            bool s_there = false;
            while (b < stop) {
              uint32_t sa[32], sb[32], pk[32];
              uint64_t sum[2] = {0, 0};
              const uint64_t mu = pack_f32x2(-m_ref, -m_ref);
              ok = __all_sync(0xffffffffu, s_there) || wait_warp(bar(ln.s_full), cnt & 1);
              if (!ok) break;
              tc_fence_after();
              tmem_ld32(cS, sa);
              tmem_ld_wait();
              tmem_ld32(cS + 32, sb);
              weights<0>(sa, sc, mu, sum, pk);
              tmem_ld_wait();
              tmem_ld32(cS + 64, sa);
              const bool o_there = peek(bar(ln.o_ready), (cnt - 1) & 1);
              weights<16>(sb, sc, mu, sum, pk);
              tmem_ld_wait();
              tmem_ld32(cS + 96, sb);
              if (cnt >= 1) {  // the P buffer was last read by the previous PV
                ok = __all_sync(0xffffffffu, o_there) || wait_warp(bar(ln.o_ready), (cnt - 1) & 1);
                if (!ok) break;
                tc_fence_after();
              }
              tmem_st32(cP, pk);
              float l0 = sum_of(sum);
              tmem_ld_wait();
              if (__any_sync(0xffffffffu, !(l0 < 0x1p60f))) {  // done anew below
                tmem_st_wait();  // over the same columns: stores of one warp keep no order by themselves
                break;
              }
              tc_fence_before();
              mbar_arrive_e(bar(ln.s_free));
              sum[0] = sum[1] = 0;
              weights<0>(sa, sc, mu, sum, pk);
              weights<16>(sb, sc, mu, sum, pk);
              float l1 = sum_of(sum);
              if (__any_sync(0xffffffffu, !(l0 + l1 < 256.f))) {
                // some rows' reference rises by a whole number of octaves, so that scaling P is exact
                float up = 0.f;
                if (!(l0 + l1 < 256.f))
                  up = fmaxf(0.f, ceilf(fmaxf(__log2f(l0), fmaxf(scores_max(sa), scores_max(sb)) * p.scale_log2 - m_ref)));
                const float f = __uint_as_float((127u - min((uint32_t)up, 127u)) << 23);  // 2^-up, 0 from 2^-127 on
                m_ref += up;
                l *= f;
                l0 *= f;
                sum[0] = sum[1] = 0;  // the second half anew: its weights may have been infinite
                weights<0>(sa, sc, pack_f32x2(-m_ref, -m_ref), sum, pk);
                weights<16>(sb, sc, pack_f32x2(-m_ref, -m_ref), sum, pk);
                l1 = sum_of(sum);
                __syncwarp();
                tmem_st_wait();
#pragma unroll 1
                for (int h = 0; h < 3; ++h) {  // P of the first half, and O
                  const uint32_t at = h ? cO + 32 * (h - 1) : cP;
                  tmem_ld32(at, sa);
                  tmem_ld_wait();
#pragma unroll
                  for (int e = 0; e < 32; ++e) {
                    const float2 w = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&sa[e]));
                    sa[e] = h ? __float_as_uint(__uint_as_float(sa[e]) * f) : pack_bf16x2(w.x * f, w.y * f);
                  }
                  __syncwarp();
                  tmem_st32(at, sa);
                }
              }
              tmem_st32(cP + 32, pk);
              const bool s_next = peek(bar(ln.s_full), (cnt + 1) & 1);
              l += l0 + l1;
              tmem_st_wait();
              tc_fence_before();
              __syncwarp();
              mbar_arrive_e(bar(ln.p_full));
              ++b, ++cnt, kb += kBlockKeys;
              s_there = s_next;
            }
            if (!ok || b == n) break;
          }
        general:
          // ---- any other block: a chunk at a time in loops that are not
          // unrolled (in a short window every block comes this way, and its
          // time is that of fetching the code)
          const bool masked = kb > plain_hi || kb < plain_lo;
          const bool dead = masked && dead_slot(a, ln.meta[slot], kb + row);
          ok = wait_warp(bar(ln.s_full), cnt & 1);
          if (!ok) break;
          // the P buffer was last read by the previous PV
          if (cnt >= 1) {
            ok = wait_warp(bar(ln.o_ready), (cnt - 1) & 1);
            if (!ok) break;
          }
          tc_fence_after();
          uint32_t sv[32], pk[32];
          auto scores = [&](int c) -> bool {  // chunk c, what is not seen at -inf; false if no row sees any of it
            const uint32_t seen = masked ? seen_keys(p, a, ln.meta[slot], my_node, kb + 32 * c) : 0xffffffffu;
            if (!__any_sync(0xffffffffu, seen != 0u)) return false;
            tmem_ld32(cS + 32 * c, sv);
            tmem_ld_wait();
            hide(sv, seen);
            return true;
          };
          const float m_start = m_ref;
          float lb;  // the block's sum
          bool redo = false;
          for (;;) {  // at most twice
            const uint64_t sc = pack_f32x2(p.scale_log2, p.scale_log2);
            uint64_t sum[2] = {0, 0};
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              __syncwarp();  // TMEM moves need the warp in step
              if (scores(c)) {
                if (unset) {  // a row's reference is the maximum of the first chunk it sees something of
                  const float mx = scores_max(sv) * p.scale_log2;
                  if (m_ref == -INFINITY) m_ref = mx;
                }
                const float neg_mu = m_ref == -INFINITY ? 0.f : -m_ref;
                weights<0>(sv, sc, pack_f32x2(neg_mu, neg_mu), sum, pk);
              } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) pk[e] = 0u;
              }
              __syncwarp();
              tmem_st16<0>(cP + 16 * c, pk);
            }
            lb = sum_of(sum);
            if (redo || !__any_sync(0xffffffffu, !(lb < 256.f))) break;
            // far beyond the reference: it becomes the block's maximum, and the block is done anew
            redo = true;
            float mx = -INFINITY;
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
              __syncwarp();
              if (scores(c)) mx = fmaxf(mx, scores_max(sv));
            }
            mx *= p.scale_log2;
            if (!(lb < 256.f) && mx > m_ref) m_ref = mx;
            __syncwarp();
            tmem_st_wait();
          }
          const float alpha = m_ref == m_start ? 1.f : ex2_approx(m_start - m_ref);  // of what earlier blocks left
          tc_fence_before();
          __syncwarp();
          mbar_arrive_e(bar(ln.s_free));
          l = l * alpha + lb;
          ok = clear_dead(dead);
          if (!ok) break;
          if (b > 0 && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              __syncwarp();
              tmem_ld32(cO + 32 * h, sv);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 32; ++e) sv[e] = __float_as_uint(__uint_as_float(sv[e]) * alpha);
              tmem_st32(cO + 32 * h, sv);
            }
          }
          unset = __any_sync(0xffffffffu, m_ref == -INFINITY);
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          mbar_arrive_e(bar(ln.p_full));
        }
      }
      if (!ok) break;
      // ---- end of the part: O / l and the log-sum-exp. O and the part's slot are
      // free for the next part as soon as they are in registers, before anything
      // is written (window of 128 keys: 97 -> 93 us). All warps load O, those
      // without rows too: a condition here costs the loops above registers.
      const bool writes = busy && tok < a.n_tok;
      const int h = a.kvh * g + head;
      const float sink = ln.meta[slot].sinks[head];
      // nothing seen: l is 0; a NaN among what is seen: l is NaN, and so are O and the log-sum-exp
      float inv = l == 0.f ? 0.f : __fdividef(1.f, l);  // l < 2^8 keys: within its range, 2 ulp
      float lse2 = l == 0.f ? -INFINITY : m_ref + __log2f(l);
      if (a.slot < 0 && sink > -INFINITY) inv = finish_with_sink(m_ref, l, sink, &lse2);
      __syncwarp();
      ok = wait_warp(bar(ln.o_ready), (cnt - 1) & 1);
      if (!ok) break;
      tc_fence_after();
      uint32_t ov[2][32];
      tmem_ld32(cO, ov[0]);
      tmem_ld32(cO + 32, ov[1]);
      tmem_ld_wait();
      tc_fence_before();
      __syncwarp();
      mbar_arrive_e(bar(ln.o_free));
      mbar_arrive_e(bar(ln.part_empty[slot]));
      const size_t orow = (size_t)(a.token + tok) * Hq + h, prow = (size_t)max(a.slot, 0) * kTileRows + row;
      if (writes && a.slot < 0) {
        uint4* dst = reinterpret_cast<uint4*>(p.out + orow * kHeadDim);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t o[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t(&v)[32] = ov[k >> 2];
            const int i = 8 * (k & 3) + 2 * e;
            o[e] = pack_bf16x2(__uint_as_float(v[i]) * inv, __uint_as_float(v[i + 1]) * inv);
          }
          dst[k] = make_uint4(o[0], o[1], o[2], o[3]);
        }
        p.lse[orow] = lse2 * 0.69314718055994531f;
      } else if (writes) {
        float4* dst = reinterpret_cast<float4*>(p.o_part + prow * kHeadDim);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const uint32_t(&v)[32] = ov[k >> 3];
          const int i = 4 * (k & 7);
          dst[k] = make_float4(__uint_as_float(v[i]) * inv, __uint_as_float(v[i + 1]) * inv,
                               __uint_as_float(v[i + 2]) * inv, __uint_as_float(v[i + 3]) * inv);
        }
        p.lse_part[prow] = lse2;
      }
    }
    if (!ok && *abort_flag == 0) *abort_flag = 1;
  }

  __syncwarp();
  if (threadIdx.x == 0 && *abort_flag == 1) atomicOr(p.status, kStatusTimeout);
  leave();
}

// Joins the parts of the tiles that cross a cut of their line: out = sum_i 2^(b_i - b) o_i,
// b = log2 sum_i 2^(b_i), in the order of the pieces. Blocks (c, y): the tile
// whose first part lies in piece c and its next ones in the pieces after it, if
// there is one (on the joint line c counts both tiles of a pair), rows 32 y ..
// of it; a thread takes four dims of a row, kMergeBatch parts' loads in flight
// at once.
constexpr int kMergeThreads = 256, kMergeRows = 32, kMergeBatch = 4;

__global__ void __launch_bounds__(kMergeThreads) merge_tree_kernel(const TreeParams p, int ctas) {
  grid_dep_wait();
  const int line = (int)blockIdx.x >= 2 * ctas, rel = (int)blockIdx.x - (line ? 2 * ctas : 0);
  const int k0 = line ? rel >> 1 : rel, x = line ? rel & 1 : 0;
  const int g = p.group, Hq = p.num_q_heads;
  const int4 cut = p.cuts[blockIdx.x];  // last piece, first token, tokens, kv head
  const int c1 = cut.x, rows = cut.z * g, kvh = cut.w;
  auto part_row = [&](int k, int r) -> size_t {
    const int first = k == k0;
    return (size_t)(line ? kTreeSoloSlots + (2 * k + first) * 2 + x : 2 * k + first) * kTileRows + r;
  };
  if (c1 <= k0) return;
  for (int v = threadIdx.x; v < kMergeRows * 16; v += kMergeThreads) {
    const int r = kMergeRows * blockIdx.y + (v >> 4), d = v & 15;
    if (r >= rows) break;
    const int h = kvh * g + r % g;
    float m = tree_sink(p, h), sum = m > -INFINITY ? 1.f : 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k = k0; k <= c1; k += kMergeBatch) {
      float b[kMergeBatch];
      float4 q[kMergeBatch];
#pragma unroll
      for (int e = 0; e < kMergeBatch; ++e) {
        b[e] = -INFINITY;
        q[e] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (k + e <= c1) {
          const size_t pr = part_row(k + e, r);
          b[e] = p.lse_part[pr];
          q[e] = reinterpret_cast<const float4*>(p.o_part + pr * kHeadDim)[d];
        }
      }
#pragma unroll
      for (int e = 0; e < kMergeBatch; ++e) {
        if (b[e] == -INFINITY) continue;
        const float mn = fmaxf(m, b[e]), f = m > -INFINITY ? exp2f(m - mn) : 0.f, wt = exp2f(b[e] - mn);
        m = mn;
        sum = sum * f + wt;
        o.x = o.x * f + wt * q[e].x;
        o.y = o.y * f + wt * q[e].y;
        o.z = o.z * f + wt * q[e].z;
        o.w = o.w * f + wt * q[e].w;
      }
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;  // a part's NaN reaches the sum, and stays
    const size_t orow = (size_t)(cut.y + r / g) * Hq + h;
    reinterpret_cast<uint2*>(p.out + orow * kHeadDim)[d] =
        make_uint2(pack_bf16x2(o.x * inv, o.y * inv), pack_bf16x2(o.z * inv, o.w * inv));
    if (d == 0) p.lse[orow] = sum == 0.f ? -INFINITY : (m + __log2f(sum)) * 0.69314718055994531f;
  }
}

}  // namespace

cudaError_t launch_tree(const CUtensorMap& kmap, const CUtensorMap& vmap, const CUtensorMap& qmap,
                        const TreeParams& p, int sms, cudaStream_t stream) {
  const int grid = sms < kTreeMaxCtas ? sms : kTreeMaxCtas;
  LaunchCfg tc(dim3(grid), dim3(kTreeThreads), tree_smem_bytes(), stream, true);
  const cudaError_t e = cudaLaunchKernelEx(&tc.cfg, tree_kernel, kmap, vmap, qmap, p);
  if (e != cudaSuccess) return e;
  // Rows whose tables, or windows, hold no more than kWholeBlocks blocks have no
  // cut tiles, and nothing to merge: without the second launch four short rows
  // take 9.3 us instead of 11.7. (The host knows the table's width, not the lengths.)
  const int64_t most_nodes = p.total_q < 32 * p.words ? p.total_q : 32 * p.words;
  int64_t keys = (int64_t)p.max_pages * kPage;
  if (p.window > 0 && keys > most_nodes + p.window + kPage) keys = most_nodes + p.window + kPage;
  if (keys <= kWholeBlocks * kBlockKeys) return cudaSuccess;
  LaunchCfg lc(dim3(4 * grid, kTileRows / kMergeRows), dim3(kMergeThreads), 0, stream, true);
  return cudaLaunchKernelEx(&lc.cfg, merge_tree_kernel, p, grid);
}

cudaError_t prepare_tree_kernels() {
  const cudaError_t e =
      cudaFuncSetAttribute(tree_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tree_smem_bytes());
  if (e != cudaSuccess) return e;
  return cudaFuncSetAttribute(tree_kernel, cudaFuncAttributePreferredSharedMemoryCarveout,
                              cudaSharedmemCarveoutMaxShared);
}

}  // namespace mcpu
