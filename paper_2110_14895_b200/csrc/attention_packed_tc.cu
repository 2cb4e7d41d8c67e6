// Attention over packed sequences on the 5th-generation tensor cores (bf16), forward and backward, for
// sequences of any length and head sizes 16 ... 128.
//
// Operands are fetched by TMA through three-dimensional maps (channel of the head, head, row) in slabs of
// 64 channels, 128-byte swizzled; channels beyond the head come as zeros, so that one layout serves every
// head size and the products run over the head's own channels only.  Scores and accumulators live in
// tensor memory; probabilities (and the scores' gradients) are written back over the scores as packed bf16
// and are the A operand of the second products, so that nothing of the score matrix leaves the SM.  One
// thread owns one row of a tile of scores.
//
// Persistent blocks, one per SM, walk over the work with a static schedule; the operands of the next piece
// are fetched while the last one is finished.  A tile of queries (or of whatever stays) is held in tensor
// memory too where it fits, as the A operand of the scores: with both operands in shared memory a product
// of 128 x 64 x 16 reads 6 KB there in the 32 cycles that it takes, more than the 128 bytes a cycle that
// shared memory gives, and holds up everything else that goes through it.
//
// Every mbarrier wait is bounded; on expiry the block raises the device status word, lets the copies and
// products in flight finish (bounded), frees tensor memory and leaves.
#include "vit_internal.h"
#include "attention_packed.cuh"
#include "sm100_ptx.cuh"

#include <cuda.h>

namespace vit {

namespace {

using namespace ptx;

constexpr int RT = 128;                                // rows of a tile of scores = lanes of tensor memory
constexpr int CT = 64;                                 // columns of a tile of scores
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;
constexpr long long DRAIN_LIMIT_CYCLES = 1ll << 24;    // teardown after a failed wait: ~10 ms
constexpr long long LONG_WAIT_CYCLES = WAIT_LIMIT_CYCLES << 8;   // for other pieces, whose own waits are bounded

// Shared-memory matrix descriptor of a 128-byte-swizzled slab (rows of 128 bytes, groups of 8 rows 1024
// bytes apart).  lbo: distance of the slabs of 64 columns, for an operand whose rows are the summed index
// (K) and that is wider than one slab.
__device__ __forceinline__ uint64_t desc_sw128(uint32_t saddr, uint32_t lbo = 16) {
  return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)((lbo >> 4) & 0x3FFFu) << 16) | ((uint64_t)(1024 >> 4) << 32) |
         ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ uint32_t idesc(int n, bool b_rows_are_k) {
  return (1u << 4) | (1u << 7) | (1u << 10) | (b_rows_are_k ? (1u << 16) : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(RT >> 4) << 24);
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* tm, int c, int head, int row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(c), "r"(head), "r"(row), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void store_16_bf16(bf16* dst, const uint32_t (&o)[16], float by) {   // 32 bytes, one sector
  uint32_t w[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = pack_bf16(__uint_as_float(o[2 * i]) * by, __uint_as_float(o[2 * i + 1]) * by);
  *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(dst + 8) = make_uint4(w[4], w[5], w[6], w[7]);
}
// a bounded wait of a whole warp: all lanes leave with the same answer
__device__ __forceinline__ bool warp_wait(uint32_t bar, int parity, volatile int* abort_flag, long long limit = WAIT_LIMIT_CYCLES) {
  return __all_sync(0xffffffffu, mbar_wait_limit(bar, (uint32_t)parity, abort_flag, limit));
}
// the same without letting the hardware suspend the warp: for the warps that issue the products, which
// otherwise take a few hundred cycles to come back
__device__ __forceinline__ bool mbar_test(uint32_t bar, int parity) {
  uint32_t done;
  asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
               : "=r"(done) : "r"(bar), "r"((uint32_t)parity) : "memory");
  return done != 0;
}
__device__ __forceinline__ bool warp_spin(uint32_t bar, int parity, volatile int* abort_flag) {
  if (__all_sync(0xffffffffu, mbar_test(bar, parity))) return true;
  const long long t0 = clock64();
  for (;;) {
    if (__all_sync(0xffffffffu, mbar_test(bar, parity))) return true;
    const bool late = clock64() - t0 > WAIT_LIMIT_CYCLES;
    if (late) *abort_flag = 1;
    if (__any_sync(0xffffffffu, late || *abort_flag)) return false;
  }
}
// rows [from, rows) of a tile of `slabs` slabs become zero; one warp, then visible to the tensor core
__device__ __forceinline__ void zero_rows(uint32_t tile, int rows, int slabs, int from, int lane) {
  for (int s = 0; s < slabs; ++s)
    for (int i = from * 8 + lane; i < rows * 8; i += 32)
      asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (uint32_t)(s * rows * 128 + i * 16)), "r"(0u) : "memory");
  fence_proxy_async_smem();
  __syncwarp();
}

// One lane of the warp, chosen by the hardware.  The products are issued behind this and not behind
// `lane == 0`: their operands then stay in uniform registers (110 -> about 20 cycles to issue one).
__device__ __forceinline__ bool elect_one() {
  uint32_t one;
  asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}\n" : "=r"(one));
  return one != 0;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }

// S[128 x n] = X[128 rows] . Y[n rows]^T over the head's channels; X in tensor memory (packed pairs) or in
// shared memory, as slabs of 64 channels like Y
template <int SLABS>
__device__ __forceinline__ void issue_scores_ts(uint32_t d_tmem, uint32_t x_tmem, uint32_t y, int n, int ksteps) {
  const uint32_t id = idesc(n, false);
  const uint64_t yd = desc_sw128(y);
#pragma unroll
  for (int k = 0; k < 4 * SLABS; ++k)
    if (k < ksteps) umma_bf16_ts(d_tmem, x_tmem + (uint32_t)(8 * k), yd + (uint64_t)((k >> 2) * (CT * 8) + 2 * (k & 3)), id, k > 0 ? 1u : 0u);
}
template <int SLABS>
__device__ __forceinline__ void issue_scores_ss(uint32_t d_tmem, uint32_t x, uint32_t y, int n, int ksteps) {
  const uint32_t id = idesc(n, false);
  const uint64_t xd = desc_sw128(x), yd = desc_sw128(y);
#pragma unroll
  for (int k = 0; k < 4 * SLABS; ++k)
    if (k < ksteps)
      umma_bf16(d_tmem, xd + (uint64_t)((k >> 2) * (RT * 8) + 2 * (k & 3)), yd + (uint64_t)((k >> 2) * (CT * 8) + 2 * (k & 3)), id,
                k > 0 ? 1u : 0u);
}
// D[128 x d] (+)= P[128 x 16 ksteps] . Y[16 ksteps rows x d], P packed in tensor memory
__device__ __forceinline__ void issue_weighted(uint32_t d_tmem, uint32_t p_tmem, uint32_t y, int d, int ksteps, bool first) {
  const uint32_t id = idesc(d, true);
  const uint64_t yd = desc_sw128(y, CT * 128);
#pragma unroll
  for (int k = 0; k < CT / 16; ++k)
    if (k < ksteps) umma_bf16_ts(d_tmem, p_tmem + (uint32_t)(8 * k), yd + (uint64_t)(k * 128), id, first && k == 0 ? 0u : 1u);
}
// The 16 channels 16 g ... of a row of a swizzled tile of 128 rows in shared memory
__device__ __forceinline__ void read_16(uint32_t (&w)[8], uint32_t tile, int row, int g) {
  const uint32_t at = tile + (uint32_t)((g >> 2) * RT * 128 + row * 128);
  const int c = 2 * (g & 3), x = row & 7;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + (uint32_t)((c ^ x) << 4)));
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "r"(at + (uint32_t)(((c + 1) ^ x) << 4)));
}
// A row of a tile from shared memory into tensor memory.  Rows behind the end of a sequence bring whatever lies
// there: every row of a product depends on its own row of this operand only.
template <int SLABS>
__device__ __forceinline__ void row_to_tmem(uint32_t taddr, uint32_t tile, int row, int d) {
#pragma unroll
  for (int g = 0; g < 4 * SLABS; ++g)
    if (g < d / 16) {
      uint32_t w[8];
      read_16(w, tile, row, g);
      tmem_st8(taddr + (uint32_t)(8 * g), w);
    }
}
__device__ __forceinline__ float dot2(uint32_t a, uint32_t b, float acc) {
  acc = fmaf(__uint_as_float(a << 16), __uint_as_float(b << 16), acc);
  return fmaf(__uint_as_float(a & 0xffff0000u), __uint_as_float(b & 0xffff0000u), acc);
}

// 64 accumulator columns of a row (those below d) times a factor to global memory: all loads, one wait, the stores
__device__ __forceinline__ void store_row(bf16* dst, uint32_t taddr, int left, float by, bool there) {
  uint32_t o[4][16];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (16 * e < left) tmem_ld16(taddr + (uint32_t)(16 * e), o[e]);
  tmem_ld_wait();
#pragma unroll
  for (int e = 0; e < 4; ++e) asm volatile("" : "+r"(o[e][0]), "+r"(o[e][1]), "+r"(o[e][2]), "+r"(o[e][3]), "+r"(o[e][4]), "+r"(o[e][5]),
      "+r"(o[e][6]), "+r"(o[e][7]), "+r"(o[e][8]), "+r"(o[e][9]), "+r"(o[e][10]), "+r"(o[e][11]), "+r"(o[e][12]), "+r"(o[e][13]),
      "+r"(o[e][14]), "+r"(o[e][15]));                           // nothing reads them before the wait
  if (!there) return;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (16 * e < left) store_16_bf16(dst + 16 * e, o[e], by);
}

// The sequences' offsets are kept in shared memory where they fit: every role of a block looks at them for every piece.
constexpr int MAX_STAGED = 1024;
constexpr uint32_t OFFSETS_BYTES = 2 * (MAX_STAGED + 1) * 4 + 8;
__device__ __forceinline__ void stage_offsets(vit_attention_problem& p, int32_t* to) {
  if (p.sequences > MAX_STAGED) return;
  for (int i = threadIdx.x; i <= p.sequences; i += (int)blockDim.x) {
    to[i] = p.q_offsets[i];
    to[MAX_STAGED + 1 + i] = p.k_offsets[i];
  }
  p.q_offsets = to;
  p.k_offsets = to + MAX_STAGED + 1;
}

// A piece of work: `span` rows of one head of one sequence.
struct Piece { int head, x0; SeqRange r; };
// The first piece from number i on (in steps of the grid) whose rows exist; i = total if there is none.
__device__ __forceinline__ int find_piece(const vit_attention_problem& p, int* status, int i, int total, int tiles, int heads, int span,
                                          bool of_keys, Piece& w) {
  for (; i < total; i += (int)gridDim.x) {
    const unsigned hs = (unsigned)i / (unsigned)tiles, seq = hs / (unsigned)heads;
    w.head = (int)(hs - seq * (unsigned)heads);
    w.x0 = (int)((unsigned)i - hs * (unsigned)tiles) * span;
    if (seq_range(p, (int)seq, w.r, status) && w.x0 < (of_keys ? w.r.k_len : w.r.q_len)) return i;
  }
  return total;
}

// ============================================================================================ forward
// A piece is 256 queries of a head: warps 0-3 and 4-7 hold 128 of them each and share the keys, which come
// in tiles of 64; warps 8 and 9 issue the products of one warpgroup each, warp 10 the copies.  Each warpgroup has two tiles of scores, so
// that the next one is ready when it has finished its exp2 phase.  The accumulator is rescaled only when a
// row's maximum has grown by more than 2^8 since the last time (probabilities stay below 2^8, the row sum
// in fp32): it rarely is after the first tile, and only then does a warpgroup wait for its last product.
struct ForwardMaps { CUtensorMap q, k, v; };

template <int SLABS, bool XT>
struct ForwardCfg {
  static constexpr int STAGES = SLABS == 1 ? 6 : 4;
  static constexpr uint32_t TILE = SLABS * CT * 128, QTILE = SLABS * RT * 128;
  static constexpr uint32_t OFF_K = 2 * QTILE, OFF_V = OFF_K + STAGES * TILE, OFF_BARS = OFF_V + STAGES * TILE, OFF_SEQ = OFF_BARS + 512;
  static constexpr uint32_t BYTES = OFF_SEQ + OFFSETS_BYTES + 1024;
  static_assert(BYTES <= 227 * 1024, "fits an SM");
};
constexpr int TC_THREADS = 384, MMA_WARP = 8 /* two */, TMA_WARP = 10;   // warp 11 only hands its registers on
// 168 registers a thread at launch (384 x 168 = 64512): the score warps take 200, the other four warps keep 96
// (256 x 200 + 128 x 96 = 63488)
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 200;"); }
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 96;"); }
constexpr uint32_t TMEM_ALL = 512;
// columns of a warpgroup (256): two tiles of scores, the accumulator (d), the queries (d / 2)
constexpr uint32_t F_WG = 256, F_O = 2 * CT;
enum FwdBar : int {
  F_KFULL = 0, F_KFREE = F_KFULL + 6, F_VFULL = F_KFREE + 6, F_VFREE = F_VFULL + 6, F_QFULL = F_VFREE + 6 /* [wg] shared memory */,
  F_QFREE = F_QFULL + 2, F_Q = F_QFREE + 2 /* [wg] tensor memory */, F_S = F_Q + 2 /* [wg][tile parity] */, F_P = F_S + 4, F_PV = F_P + 4, F_DRAIN = F_PV + 4 /* [MMA warp] */, F_BARS = F_DRAIN + 2
};

template <int SLABS, bool XT>
__global__ void __launch_bounds__(TC_THREADS, 1)
packed_forward_tc_kernel(const __grid_constant__ ForwardMaps maps, const PackedCall c, int total, int tiles) {
  using L = ForwardCfg<SLABS, XT>;
  extern __shared__ uint8_t smem_raw[];
  const int d = c.p.d, group = c.p.heads / c.p.kv_heads;
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sb = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BARS);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(&bars[F_BARS]);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < F_BARS; ++i) {
      const bool stage_free = (i >= F_KFREE && i < F_KFREE + 6) || (i >= F_VFREE && i < F_VFREE + 6);   // by both MMA warps
      const bool by_warps = (i >= F_P && i < F_P + 4) || i == F_Q || i == F_Q + 1 || (XT && (i == F_QFREE || i == F_QFREE + 1));
      mbar_init(bar(i), stage_free ? 2 : by_warps ? 4 : 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == MMA_WARP) tmem_alloc(smem_u32(tmem_slot), TMEM_ALL);
  vit_attention_problem p = c.p;
  stage_offsets(p, reinterpret_cast<int32_t*>(smem + L::OFF_SEQ));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  Piece w;
  auto find = [&](int i) { return find_piece(p, c.dev_status, i, total, tiles, p.heads, 2 * RT, false, w); };

  if (warp >= MMA_WARP) give_registers();
  else take_registers();
  if (warp > TMA_WARP) {
  } else if (warp == TMA_WARP) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int t = 0, q_tiles[2] = {0, 0}, armed_k = 0, armed_v = 0;   // tiles of keys and of queries so far
      bool ok = true;
      for (int i = find(blockIdx.x); i < total && ok; i = find(i + gridDim.x)) {
        const int n = (w.r.k_len + CT - 1) / CT, kv = w.head / group;
        if (n == 0) continue;
        for (int h = 0; h < 2 && ok; ++h) {
          if (w.x0 + h * RT >= w.r.q_len) break;
          if (!mbar_wait_limit(bar(F_QFREE + h), (q_tiles[h] & 1) ^ 1, abort_flag, LONG_WAIT_CYCLES)) { ok = false; break; }
          mbar_arrive_expect_tx(bar(F_QFULL + h), L::QTILE);
          ++q_tiles[h];
          for (int s = 0; s < SLABS; ++s)
            tma_load_3d(sb + h * L::QTILE + s * RT * 128, &maps.q, 64 * s, w.head, w.r.q_begin + w.x0 + h * RT, bar(F_QFULL + h));
        }
        for (int j = 0; j < n && ok; ++j, ++t) {
          const int st = t % L::STAGES, ph = (t / L::STAGES) & 1, krow = w.r.k_begin + j * CT;
          if (!mbar_wait(bar(F_KFREE + st), ph ^ 1, abort_flag)) { ok = false; break; }
          mbar_arrive_expect_tx(bar(F_KFULL + st), L::TILE);
          armed_k = t + 1;
          for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + L::OFF_K + st * L::TILE + s * CT * 128, &maps.k, 64 * s, kv, krow, bar(F_KFULL + st));
          if (!mbar_wait(bar(F_VFREE + st), ph ^ 1, abort_flag)) { ok = false; break; }
          mbar_arrive_expect_tx(bar(F_VFULL + st), L::TILE);
          armed_v = t + 1;
          for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + L::OFF_V + st * L::TILE + s * CT * 128, &maps.v, 64 * s, kv, krow, bar(F_VFULL + st));
        }
      }
      if (*abort_flag) {
        // a wait gave up somewhere: let the copies that were started land before the block leaves
        volatile int never = 0;
        for (int h = 0; h < 2; ++h)
          if (q_tiles[h]) mbar_wait_limit(bar(F_QFULL + h), (q_tiles[h] - 1) & 1, &never, DRAIN_LIMIT_CYCLES);
        for (int i = armed_k > L::STAGES ? armed_k - L::STAGES : 0; i < armed_k; ++i)
          mbar_wait_limit(bar(F_KFULL + i % L::STAGES), (i / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
        for (int i = armed_v > L::STAGES ? armed_v - L::STAGES : 0; i < armed_v; ++i)
          mbar_wait_limit(bar(F_VFULL + i % L::STAGES), (i / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
      }
    }
  } else if (warp >= MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuers, one per warpgroup (the whole warp keeps step)
    const int h = warp - MMA_WARP;
    const uint32_t base = tmem + h * F_WG;
    int t0 = 0, g = 0, seen = 0;                                 // tiles of keys so far, those of this warpgroup, pieces
    bool ok = true;
    for (int i = find(blockIdx.x); i < total && ok; i = find(i + gridDim.x)) {
      const int n = (w.r.k_len + CT - 1) / CT;
      if (n == 0) continue;
      const bool mine = w.x0 + h * RT < w.r.q_len;               // else the stages are passed on only
      for (int j = 0; j <= n; ++j) {
        if (j < n) {
          const int st = (t0 + j) % L::STAGES, n16 = (min(CT, w.r.k_len - j * CT) + 15) / 16, b = (g + j) & 1;
          const uint32_t ks = sb + L::OFF_K + st * L::TILE;
          if (!warp_spin(bar(F_KFULL + st), ((t0 + j) / L::STAGES) & 1, abort_flag)) { ok = false; break; }
          if (j == 0 && mine && !warp_spin(bar((XT ? F_Q : F_QFULL) + h), seen & 1, abort_flag)) { ok = false; break; }
          if (elect_one()) {
            if (mine) {
              // the scores overwrite P of tile j - 2: its product was issued before, by this warp
              tc_fence_after();
              if (XT) issue_scores_ts<SLABS>(base + b * CT, base + F_O + d, ks, 16 * n16, d / 16);
              else issue_scores_ss<SLABS>(base + b * CT, sb + h * L::QTILE, ks, 16 * n16, d / 16);
              umma_commit(bar(F_S + 2 * h + b));
              if (!XT && j == n - 1) umma_commit(bar(F_QFREE + h));
            }
            umma_commit(bar(F_KFREE + st));
          }
          __syncwarp();                                          // lanes that poll would hold up the one that issues
        }
        if (j > 0) {
          const int jj = j - 1, st = (t0 + jj) % L::STAGES, here = min(CT, w.r.k_len - jj * CT), n16 = (here + 15) / 16, b = (g + jj) & 1;
          const uint32_t vs = sb + L::OFF_V + st * L::TILE;
          if (!warp_spin(bar(F_VFULL + st), ((t0 + jj) / L::STAGES) & 1, abort_flag)) { ok = false; break; }
          // rows of V behind the last key meet probabilities of zero: make them zero too, whatever lies there
          // (both warps write the same zeros; neither reads before its own are there)
          if (mine && here < 16 * n16) zero_rows(vs, CT, SLABS, here, lane);
          if (mine && !warp_spin(bar(F_P + 2 * h + b), ((g + jj) >> 1) & 1, abort_flag)) { ok = false; break; }
          if (elect_one()) {
            if (mine) {
              tc_fence_after();
              issue_weighted(base + F_O, base + b * CT, vs, d, n16, jj == 0);
              umma_commit(bar(F_PV + 2 * h + b));
            }
            umma_commit(bar(F_VFREE + st));
          }
          __syncwarp();
        }
      }
      t0 += n;
      if (mine) {
        ++seen;
        g += n;
      }
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      volatile int never = 0;
      umma_commit(bar(F_DRAIN + h));
      mbar_wait_limit(bar(F_DRAIN + h), 0, &never, DRAIN_LIMIT_CYCLES);
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    const int wg = warp >> 2, in_tile = (warp & 3) * 32 + lane;
    const uint32_t taddr = tmem + ((uint32_t)((warp & 3) * 32) << 16) + wg * F_WG;
    const float sl2 = c.p.scale * LOG2E;
    const float2 sl2v = make_float2(sl2, sl2);
    // the next piece that has keys and rows for this warpgroup; queries without keys are finished on the way
    auto next = [&](int i) {
      for (i = find(i); i < total; i = find(i + gridDim.x)) {
        if (w.x0 + wg * RT >= w.r.q_len) continue;
        if (w.r.k_len > 0) break;
        const int row = w.x0 + wg * RT + in_tile;
        if (row < w.r.q_len) {
          const int64_t at = (int64_t)w.r.q_begin + row;
          bf16* out = static_cast<bf16*>(c.out) + at * c.ldo + (int64_t)w.head * d;
          for (int e = 0; e < d; e += 8) *reinterpret_cast<uint4*>(out + e) = make_uint4(0u, 0u, 0u, 0u);
          c.lse[(int64_t)w.head * c.p.q_rows + at] = -INFINITY;
        }
      }
      return i;
    };
    int g = 0, seen = 0;                                         // tiles and pieces of this warpgroup so far
    // this thread's query of the next piece into tensor memory (the scores that used the last one are complete)
    auto load_query = [&] {
      if (!warp_wait(bar(F_QFULL + wg), seen & 1, abort_flag, LONG_WAIT_CYCLES)) return false;
      ++seen;
      row_to_tmem<SLABS>(taddr + F_O + d, sb + wg * L::QTILE, in_tile, d);
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(F_Q + wg));
        mbar_arrive(bar(F_QFREE + wg));
      }
      return true;
    };
    int i = next(blockIdx.x);
    bool ok = !XT || i >= total || load_query();
    while (i < total && ok) {
      const Piece now = w;
      const int n = (now.r.k_len + CT - 1) / CT, row = now.x0 + wg * RT + in_tile;
      const bool warp_active = now.x0 + wg * RT + (warp & 3) * 32 < now.r.q_len;
      float m = -INFINITY, l = 0.f;                              // row maximum in use (raw scores), row sum
      for (int j = 0; j < n; ++j, ++g) {
        const int b = g & 1, here = min(CT, now.r.k_len - j * CT);
        const uint32_t s_col = taddr + b * CT;
        // a warpgroup without rows in the pieces before this one waits for all of them: what bounds the wait is
        // the limit of the warps that are at work
        if (!warp_wait(bar(F_S + 2 * wg + b), (g >> 1) & 1, abort_flag, j == 0 ? LONG_WAIT_CYCLES : WAIT_LIMIT_CYCLES)) { ok = false; break; }
        tc_fence_after();
        if (warp_active) {
          uint32_t x[2][32];
          tmem_ld32(s_col, x[0]);
          tmem_ld32(s_col + 32, x[1]);
          tmem_ld_wait_for(x[0]);
          tmem_ld_wait_for(x[1]);
          if (here < CT) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (32 * h + e >= here) x[h][e] = 0xff800000u;   // keys behind the end: minus infinity
          }
          float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              asm("max.f32 %0, %0, %1, %2;" : "+f"(m4[2 * h]) : "f"(__uint_as_float(x[h][e])), "f"(__uint_as_float(x[h][e + 1])));
              asm("max.f32 %0, %0, %1, %2;" : "+f"(m4[2 * h + 1]) : "f"(__uint_as_float(x[h][e + 2])), "f"(__uint_as_float(x[h][e + 3])));
            }
          }
          const float top = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
          const bool grow = (top - m) * sl2 > 8.f;               // false for NaN and for -infinity over -infinity
          if (__any_sync(0xffffffffu, grow)) {
            const float factor = grow ? (m == -INFINITY ? 0.f : ex2_approx((m - top) * sl2)) : 1.f;
            if (grow) m = top;
            l *= factor;
            if (j > 0) {
              if (!warp_wait(bar(F_PV + 2 * wg + (b ^ 1)), ((g - 1) >> 1) & 1, abort_flag)) { ok = false; break; }
              tc_fence_after();
              for (int e = 0; e < d / 16; ++e) {
                uint32_t o[16];
                tmem_ld16(taddr + F_O + (uint32_t)(16 * e), o);
                tmem_ld_wait();
#pragma unroll
                for (int f = 0; f < 16; ++f) o[f] = __float_as_uint(__uint_as_float(o[f]) * factor);
                tmem_st16(taddr + F_O + (uint32_t)(16 * e), o);
              }
            }
          }
          // p = exp2((s - m) sl2), row sum, P (bf16 pairs) over the scores
          const float nm = m == -INFINITY ? 0.f : -m * sl2;
          const float2 nmv = make_float2(nm, nm);
          float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            uint32_t pk[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 y = __ffma2_rn(make_float2(__uint_as_float(x[h][2 * e]), __uint_as_float(x[h][2 * e + 1])), sl2v, nmv);
              const float2 p = make_float2(ex2_approx(y.x), ex2_approx(y.y));
              l2[e & 1] = __fadd2_rn(l2[e & 1], p);
              pk[e] = pack_bf16(p.x, p.y);
            }
            tmem_st16(s_col + (uint32_t)(16 * h), pk);
          }
          l2[0] = __fadd2_rn(l2[0], l2[1]);
          l += l2[0].x + l2[0].y;
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(F_P + 2 * wg + b));
      }
      if (!ok) break;
      i = next(i + gridDim.x);
      if (XT && i < total && !load_query()) break;
      if (!warp_wait(bar(F_PV + 2 * wg + ((g - 1) & 1)), ((g - 1) >> 1) & 1, abort_flag)) break;
      tc_fence_after();
      if (warp_active) {
        const bool there = row < now.r.q_len;
        const int64_t at = (int64_t)now.r.q_begin + row;
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        bf16* out = static_cast<bf16*>(c.out) + at * c.ldo + (int64_t)now.head * d;
#pragma unroll
        for (int s = 0; s < SLABS; ++s) store_row(out + 64 * s, taddr + F_O + 64 * s, d - 64 * s, inv, there);
        if (there) c.lse[(int64_t)now.head * c.p.q_rows + at] = l == 0.f ? -INFINITY : fmaf(m, c.p.scale, log2f(l) * LN2);
      }
    }
  }
  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(c.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == MMA_WARP) {
    __syncwarp();
    tmem_dealloc(tmem, TMEM_ALL);
  }
}

// ============================================================================================ backward
// Two kernels of one form.  A piece is a tile of 128 rows X1, X2 of a head, which stays, and tiles of 64 rows
// Y1, Y2 go by:
//   S = X1 Y1^T, dP = X2 Y2^T;  P = exp2(S sl2 - lse2), dS = P (dP - delta)
//   DQ:   X = Q, dout; Y = K, V;  dq += dS Y1.  It comes first and also writes lse2 and delta of its rows.
//   DKDV: X = K, V; Y = Q, dout of every query head that shares the key head (scores transposed);
//         dv += P Y2, dk += dS Y1
// Seven products instead of the five of a single pass, but every gradient is summed in one place in a fixed
// order.  Two warpgroups take the tiles in turn, each with its own columns of tensor memory for S and dP:
// while one is in its exp2 phase the tensor core works for the other.  X is in tensor memory (XT) where it
// fits beside the accumulators: always for DQ, up to d = 80 for DKDV.
struct BackwardMaps { CUtensorMap x1, x2, x3, y1, y2; };

template <int SLABS, bool DKDV, bool XT>
struct BackwardCfg {
  static constexpr int XS = DKDV ? 2 : 3;              // tiles of X in shared memory; DQ: out, for delta
  static constexpr int STAGES = SLABS == 1 ? 6 : DKDV ? 4 : 3;
  static constexpr uint32_t XTILE = SLABS * RT * 128, YTILE = SLABS * CT * 128;
  static constexpr uint32_t OFF_Y = XS * XTILE, OFF_COL = OFF_Y + STAGES * 2 * YTILE;   // DKDV: float [STAGES][2][64] -lse2, -delta of the columns
  static constexpr uint32_t OFF_ROW = OFF_COL + (DKDV ? STAGES * CT * 8 : 0);           // DQ: float2 [2][128] of the rows
  static constexpr uint32_t OFF_BARS = OFF_ROW + (DKDV ? 0 : 2 * RT * 8), OFF_SEQ = OFF_BARS + 512;
  static constexpr uint32_t BYTES = OFF_SEQ + OFFSETS_BYTES + 1024;
  static_assert(BYTES <= 227 * 1024, "fits an SM");
};
// columns: S and dP of the two warpgroups, then the accumulators (d each), then X1 and X2 (d / 2 each)
constexpr uint32_t B_WG = 2 * CT, B_COLS = 2 * B_WG;
enum BwdBar : int {
  B_FULL = 0, B_FREE = B_FULL + 6, B_XS = B_FREE + 6 /* X in shared memory */, B_XSFREE, B_X /* in tensor memory */, B_XFREE, B_S, B_P = B_S + 2, B_SFREE = B_P + 2, B_ACC = B_SFREE + 2, B_ACCFREE,
  B_DRAIN /* [MMA warp] */, B_BARS = B_DRAIN + 2
};

template <int SLABS, bool DKDV, bool XT>
__global__ void __launch_bounds__(TC_THREADS, 1)
packed_backward_tc_kernel(const __grid_constant__ BackwardMaps maps, const PackedCall c, int total, int tiles) {
  using L = BackwardCfg<SLABS, DKDV, XT>;
  extern __shared__ uint8_t smem_raw[];
  const int d = c.p.d, group = c.p.heads / c.p.kv_heads, x_heads = DKDV ? c.p.kv_heads : c.p.heads;
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sb = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BARS);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(&bars[B_BARS]);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < B_BARS; ++i)
      mbar_init(bar(i), i == B_P || i == B_P + 1 ? 4 : i == B_ACCFREE || i == B_X || (XT && i == B_XSFREE) ? 8 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == MMA_WARP) tmem_alloc(smem_u32(tmem_slot), TMEM_ALL);
  vit_attention_problem p = c.p;
  stage_offsets(p, reinterpret_cast<int32_t*>(smem + L::OFF_SEQ));
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);
  const uint32_t acc2 = B_COLS, acc1 = B_COLS + d, x1_col = B_COLS + (DKDV ? 2 : 1) * d, x2_col = x1_col + d / 2;   // dk or dq; dv
  Piece w;
  auto find = [&](int i) { return find_piece(p, c.dev_status, i, total, tiles, x_heads, RT, DKDV, w); };
  // tiles of Y that a piece walks over, head after head
  auto y_tiles_of = [&](const Piece& p) { return ((DKDV ? p.r.q_len : p.r.k_len) + CT - 1) / CT; };

  if (warp >= MMA_WARP) give_registers();
  else take_registers();
  if (warp > TMA_WARP) {
  } else if (warp == TMA_WARP) {
    // ------------------------------------------------------------------ producer (the whole warp keeps step)
    int t0 = 0, pieces = 0, armed = 0;
    bool ok = true;
    for (int i = find(blockIdx.x); i < total && ok; i = find(i + gridDim.x)) {
      const int y_tiles = y_tiles_of(w), n = DKDV ? group * y_tiles : y_tiles;
      const int y_begin = DKDV ? w.r.q_begin : w.r.k_begin, y_len = DKDV ? w.r.q_len : w.r.k_len;
      if (n == 0) continue;
      if (!warp_wait(bar(B_XSFREE), (pieces & 1) ^ 1, abort_flag)) break;
      if (lane == 0) {
        const int row = (DKDV ? w.r.k_begin : w.r.q_begin) + w.x0;
        mbar_arrive_expect_tx(bar(B_XS), L::XS * L::XTILE);
        for (int s = 0; s < SLABS; ++s) {
          tma_load_3d(sb + s * RT * 128, &maps.x1, 64 * s, w.head, row, bar(B_XS));
          tma_load_3d(sb + L::XTILE + s * RT * 128, &maps.x2, 64 * s, w.head, row, bar(B_XS));
          if (!DKDV) tma_load_3d(sb + 2 * L::XTILE + s * RT * 128, &maps.x3, 64 * s, w.head, row, bar(B_XS));
        }
      }
      ++pieces;
      int yt = 0, yh = DKDV ? w.head * group : w.head / group;
      for (int t = t0; t < t0 + n; ++t) {
        const int st = t % L::STAGES, ph = (t / L::STAGES) & 1, y0 = yt * CT;
        const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE;
        // DKDV: the numbers of the tile's columns travel with it, negated; beyond the sequence
        // P = exp2(0 - infinity) = 0 and dS = 0.  They are in flight while this warp waits for the stage.
        float2 v[2];
        if (DKDV) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            v[e] = make_float2(INFINITY, 0.f);
            if (y0 + 32 * e + lane < y_len) v[e] = c.delta[(int64_t)yh * c.p.q_rows + y_begin + y0 + 32 * e + lane];
          }
        }
        if (!warp_wait(bar(B_FREE + st), ph ^ 1, abort_flag)) { ok = false; break; }
        if (DKDV) {
          float* col = reinterpret_cast<float*>(smem + L::OFF_COL) + st * 2 * CT;
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            col[32 * e + lane] = -v[e].x;
            col[CT + 32 * e + lane] = -v[e].y;
          }
          __syncwarp();
        }
        armed = t + 1;
        if (lane == 0) {
          mbar_arrive_expect_tx(bar(B_FULL + st), 2 * L::YTILE);
          for (int s = 0; s < SLABS; ++s) {
            tma_load_3d(y + s * CT * 128, &maps.y1, 64 * s, yh, y_begin + y0, bar(B_FULL + st));
            tma_load_3d(y + L::YTILE + s * CT * 128, &maps.y2, 64 * s, yh, y_begin + y0, bar(B_FULL + st));
          }
        }
        if (++yt == y_tiles) { yt = 0; ++yh; }
      }
      t0 += n;
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      // a wait gave up somewhere: let the copies that were started land before the block leaves
      volatile int never = 0;
      if (pieces) mbar_wait_limit(bar(B_XS), (pieces - 1) & 1, &never, DRAIN_LIMIT_CYCLES);
      for (int t = armed > L::STAGES ? armed - L::STAGES : 0; t < armed; ++t)
        mbar_wait_limit(bar(B_FULL + t % L::STAGES), (t / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
    }
  } else if (warp >= MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuers (whole warps keep step): one of the
    // scores, one of the second products
    const bool scores = warp == MMA_WARP;
    int t0 = 0, pieces = 0;
    uint32_t phase = 0;                                          // bit b: parity of the next wait for warpgroup b's columns
    bool ok = true;
    for (int i = find(blockIdx.x); i < total && ok; i = find(i + gridDim.x)) {
      const int y_tiles = y_tiles_of(w), n = DKDV ? group * y_tiles : y_tiles, y_len = DKDV ? w.r.q_len : w.r.k_len;
      if (n == 0) continue;
      if (scores && !warp_spin(bar(XT ? B_X : B_XS), pieces & 1, abort_flag)) break;
      const int last = y_len - (y_tiles - 1) * CT;               // rows of a head's last tile
      int yt = 0;                                                // tile of its head
      for (int t = 0; t < n; ++t) {
        const int st = (t0 + t) % L::STAGES, b = t & 1, here = yt == y_tiles - 1 ? last : CT, n16 = (here + 15) / 16;
        const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE, s_col = tmem + b * B_WG;
        if (++yt == y_tiles) yt = 0;
        if (scores) {
          if (!warp_spin(bar(B_FULL + st), ((t0 + t) / L::STAGES) & 1, abort_flag)) { ok = false; break; }
          // rows of Y behind the end of the sequence become zero, whatever lies there: they meet weights of
          // zero in the second products, and give scores of zero in the first
          if (here < 16 * n16) {
            zero_rows(y, CT, SLABS, here, lane);
            zero_rows(y + L::YTILE, CT, SLABS, here, lane);
          }
          // S and dP overwrite P and dS of tile t - 2, once their products are complete
          if (!warp_spin(bar(B_SFREE + b), (phase >> b & 1) ^ 1, abort_flag)) { ok = false; break; }
          phase ^= 1u << b;
          if (elect_one()) {
            tc_fence_after();
            if (XT) {
              issue_scores_ts<SLABS>(s_col, tmem + x1_col, y, 16 * n16, d / 16);
              issue_scores_ts<SLABS>(s_col + CT, tmem + x2_col, y + L::YTILE, 16 * n16, d / 16);
            } else {
              issue_scores_ss<SLABS>(s_col, sb, y, 16 * n16, d / 16);
              issue_scores_ss<SLABS>(s_col + CT, sb + L::XTILE, y + L::YTILE, 16 * n16, d / 16);
            }
            umma_commit(bar(B_S + b));
            if (t == n - 1) umma_commit(bar(XT ? B_XFREE : B_XSFREE));
          }
        } else {
          if (!warp_spin(bar(B_P + b), phase >> b & 1, abort_flag)) { ok = false; break; }
          phase ^= 1u << b;
          // the accumulators of the last piece have been read
          if (t == 0 && !warp_spin(bar(B_ACCFREE), (pieces & 1) ^ 1, abort_flag)) { ok = false; break; }
          if (elect_one()) {
            tc_fence_after();
            if (DKDV) issue_weighted(tmem + acc1, s_col, y + L::YTILE, d, n16, t == 0);
            issue_weighted(tmem + acc2, s_col + CT, y, d, n16, t == 0);
            umma_commit(bar(B_SFREE + b));
            umma_commit(bar(B_FREE + st));
            if (t == n - 1) umma_commit(bar(B_ACC));
          }
        }
        __syncwarp();                                            // lanes that poll would hold up the one that issues
      }
      t0 += n;
      ++pieces;
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      volatile int never = 0;
      umma_commit(bar(B_DRAIN + warp - MMA_WARP));
      mbar_wait_limit(bar(B_DRAIN + warp - MMA_WARP), 0, &never, DRAIN_LIMIT_CYCLES);
    }
  } else {
    // ------------------------------------------------------------------ probabilities and their gradients
    const int wg = warp >> 2, in_tile = (warp & 3) * 32 + lane;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t taddr = lanes + wg * B_WG;
    const float sl2 = c.p.scale * LOG2E;
    const float2 sl2v = make_float2(sl2, sl2);
    int pieces = 0, t0 = 0;
    uint32_t s_phase = 0;
    bool ok = true;
    auto grad1 = [&](const Piece& p, int64_t at) { return static_cast<bf16*>(c.dv) + at * c.lddv + (int64_t)p.head * d; };
    auto grad2 = [&](const Piece& p, int64_t at) {
      return DKDV ? static_cast<bf16*>(c.dk) + at * c.lddk + (int64_t)p.head * d : static_cast<bf16*>(c.dq) + at * c.lddq + (int64_t)p.head * d;
    };
    // the next piece with something to walk over; rows that nothing meets get gradients of zero on the way
    auto next = [&](int i) {
      for (i = find(i); i < total; i = find(i + gridDim.x)) {
        if (y_tiles_of(w) > 0) break;
        const int row = w.x0 + in_tile;
        const int64_t at = (int64_t)(DKDV ? w.r.k_begin : w.r.q_begin) + row;
        if (wg == 0 && row < (DKDV ? w.r.k_len : w.r.q_len))
          for (int e = 0; e < d; e += 8) {
            *reinterpret_cast<uint4*>(grad2(w, at) + e) = make_uint4(0u, 0u, 0u, 0u);
            if (DKDV) *reinterpret_cast<uint4*>(grad1(w, at) + e) = make_uint4(0u, 0u, 0u, 0u);
          }
      }
      return i;
    };
    // this thread's row of X1 (first warpgroup) or X2 (second) of piece w into tensor memory; the second
    // warpgroup of DQ has dout and takes its product with out on the way
    auto load_x = [&] {
      if (!warp_wait(bar(B_XS), pieces & 1, abort_flag)) return false;
      row_to_tmem<SLABS>(lanes + (wg == 0 ? x1_col : x2_col), sb + wg * L::XTILE, in_tile, d);
      if (!DKDV && wg == 1) {
        const int row = w.x0 + in_tile;
        const int64_t i = (int64_t)w.head * c.p.q_rows + w.r.q_begin + row;
        const bool there = row < w.r.q_len;
        const float lse = there ? c.lse[i] : 0.f;
        float delta = 0.f;
#pragma unroll
        for (int g = 0; g < 4 * SLABS; ++g)
          if (g < d / 16) {
            uint32_t u[8], v[8];
            read_16(u, sb + L::XTILE, in_tile, g);
            read_16(v, sb + 2 * L::XTILE, in_tile, g);
#pragma unroll
            for (int e = 0; e < 8; ++e) delta = dot2(u[e], v[e], delta);
          }
        const float2 mine = make_float2(lse * LOG2E, delta);
        reinterpret_cast<float2*>(smem + L::OFF_ROW)[(pieces & 1) * RT + in_tile] = mine;
        if (there) c.delta[i] = mine;
      }
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(B_X));
        mbar_arrive(bar(B_XSFREE));
      }
      return true;
    };
    int i = next(blockIdx.x);
    ok = !XT || i >= total || load_x();
    while (i < total && ok) {
      const Piece now = w;
      const int y_tiles = y_tiles_of(now), n = DKDV ? group * y_tiles : y_tiles, y_len = DKDV ? now.r.q_len : now.r.k_len;
      const int x_len = DKDV ? now.r.k_len : now.r.q_len, row = now.x0 + in_tile;
      const bool warp_active = now.x0 + (warp & 3) * 32 < x_len;
      float2 nls = make_float2(0.f, 0.f), nde = nls;             // DQ: of this thread's row
      if (!DKDV) {
        if (!warp_wait(bar(B_X), pieces & 1, abort_flag)) break;
        const float2 mine = reinterpret_cast<const float2*>(smem + L::OFF_ROW)[(pieces & 1) * RT + in_tile];
        nls = make_float2(-mine.x, -mine.x);
        nde = make_float2(-mine.y, -mine.y);
      }
      int yt = wg % y_tiles;                                     // DKDV: tile of its head
      for (int t = wg; t < n; t += 2) {
        const int here = (DKDV ? yt : t) == y_tiles - 1 ? y_len - (y_tiles - 1) * CT : CT, nch = (here + 31) / 32;
        const int st = (t0 + t) % L::STAGES;
        const float4* col = reinterpret_cast<const float4*>(smem + L::OFF_COL) + st * (CT / 2);   // four columns each: -lse2, then -delta
        if (DKDV) {
          yt = (yt + 2) % y_tiles;
          if (!warp_wait(bar(B_FULL + st), ((t0 + t) / L::STAGES) & 1, abort_flag)) { ok = false; break; }
        }
        if (!warp_wait(bar(B_S + wg), s_phase, abort_flag)) { ok = false; break; }
        s_phase ^= 1;
        tc_fence_after();
        if (warp_active) {
          uint32_t s[2][32], g[2][32];
          tmem_ld32(taddr, s[0]);
          tmem_ld32(taddr + CT, g[0]);
          tmem_ld_wait_for(s[0]);
          tmem_ld_wait_for(g[0]);
          if (nch > 1) {
            tmem_ld32(taddr + 32, s[1]);
            tmem_ld32(taddr + CT + 32, g[1]);
          }
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h >= nch) break;
            if (h == 1) {
              tmem_ld_wait_for(s[1]);
              tmem_ld_wait_for(g[1]);
            }
            uint32_t pk[16], dk[16];
            const int left = here - 32 * h;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              float4 a4 = make_float4(nls.x, nls.x, nls.x, nls.x), b4 = make_float4(nde.x, nde.x, nde.x, nde.x);
              if (DKDV) {
                a4 = col[8 * h + q];
                b4 = col[CT / 4 + 8 * h + q];
              }
#pragma unroll
              for (int f = 0; f < 2; ++f) {
                const int e = 2 * q + f;
                const float2 a = f ? make_float2(a4.z, a4.w) : make_float2(a4.x, a4.y), b = f ? make_float2(b4.z, b4.w) : make_float2(b4.x, b4.y);
                const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[h][2 * e]), __uint_as_float(s[h][2 * e + 1])), sl2v, a);
                float2 p = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                if (!DKDV && left < 32) {                        // keys behind the end
                  if (2 * e >= left) p.x = 0.f;
                  if (2 * e + 1 >= left) p.y = 0.f;
                }
                const float2 y = __fmul2_rn(p, __fadd2_rn(make_float2(__uint_as_float(g[h][2 * e]), __uint_as_float(g[h][2 * e + 1])), b));
                if (DKDV) pk[e] = pack_bf16(p.x, p.y);
                dk[e] = pack_bf16(y.x, y.y);
              }
            }
            if (DKDV) tmem_st16(taddr + (uint32_t)(16 * h), pk);
            tmem_st16(taddr + (uint32_t)(CT + 16 * h), dk);
          }
          tmem_st_wait();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(B_P + wg));
      }
      if (!ok) break;
      t0 += n;
      ++pieces;
      i = next(i + gridDim.x);
      if (XT && i < total) {
        // every score of the last piece is complete: its X may be overwritten
        if (!warp_wait(bar(B_XFREE), (pieces - 1) & 1, abort_flag)) break;
        tc_fence_after();
        if (!load_x()) break;
      }
      if (!warp_wait(bar(B_ACC), (pieces - 1) & 1, abort_flag)) break;
      tc_fence_after();
      if (warp_active) {
        const int64_t at = (int64_t)(DKDV ? now.r.k_begin : now.r.q_begin) + row;
        const bool there = row < x_len;
        // DKDV: dk by the first warpgroup, dv by the second; DQ: halves of the head
        if (DKDV) {
          bf16* to = wg == 0 ? grad2(now, at) : grad1(now, at);
#pragma unroll
          for (int s = 0; s < SLABS; ++s) store_row(to + 64 * s, lanes + (wg == 0 ? acc2 : acc1) + 64 * s, d - 64 * s, wg == 0 ? c.p.scale : 1.f, there);
        } else {
          const int half = d / 32 * 16, from = wg == 0 ? 0 : half;
          store_row(grad2(now, at) + from, lanes + acc2 + from, wg == 0 ? half : d - half, c.p.scale, there);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_ACCFREE));
    }
  }
  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(c.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == MMA_WARP) {
    __syncwarp();
    tmem_dealloc(tmem, TMEM_ALL);
  }
}

// ============================================================================================ launches
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encoder() {
  static const EncodeTiledFn fn = [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess)
      p = nullptr;
    return reinterpret_cast<EncodeTiledFn>(p);
  }();
  return fn;
}

// (channel, head, row) of a buffer [rows, heads * d] with row stride ld; boxes of 64 channels x 1 head x box_rows rows
bool encode_heads(CUtensorMap* tm, const void* base, int64_t rows, int heads, int d, int64_t ld, int box_rows) {
  const EncodeTiledFn fn = encoder();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)rows};
  const cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)ld * 2};
  const cuuint32_t box[3] = {64, 1, (cuuint32_t)box_rows}, one[3] = {1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int SLABS, bool XT>
cudaError_t launch_forward(const PackedCall& c, cudaStream_t s) {
  using L = ForwardCfg<SLABS, XT>;
  ForwardMaps m;
  if (!encode_heads(&m.q, c.q, c.p.q_rows, c.p.heads, c.p.d, c.ldq, RT)) return cudaErrorInvalidValue;
  if (c.p.k_rows > 0) {
    if (!encode_heads(&m.k, c.k, c.p.k_rows, c.p.kv_heads, c.p.d, c.ldk, CT)) return cudaErrorInvalidValue;
    if (!encode_heads(&m.v, c.v, c.p.k_rows, c.p.kv_heads, c.p.d, c.ldv, CT)) return cudaErrorInvalidValue;
  } else {
    m.k = m.v = m.q;                                   // no keys at all: never used
  }
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_forward_tc_kernel<SLABS, XT>, (int)L::BYTES)) return e;
  const int sms = current_device_sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  const int tiles = (c.p.max_q + 2 * RT - 1) / (2 * RT), total = c.p.sequences * c.p.heads * tiles;
  packed_forward_tc_kernel<SLABS, XT><<<total < sms ? total : sms, TC_THREADS, L::BYTES, s>>>(m, c, total, tiles);
  return cudaGetLastError();
}

template <int SLABS, bool DKDV, bool XT>
cudaError_t launch_backward(const PackedCall& c, cudaStream_t s) {
  using L = BackwardCfg<SLABS, DKDV, XT>;
  BackwardMaps m;
  const void *x1 = DKDV ? c.k : c.q, *x2 = DKDV ? c.v : c.dout, *y1 = DKDV ? c.q : c.k, *y2 = DKDV ? c.dout : c.v;
  const int64_t lx1 = DKDV ? c.ldk : c.ldq, lx2 = DKDV ? c.ldv : c.lddo, ly1 = DKDV ? c.ldq : c.ldk, ly2 = DKDV ? c.lddo : c.ldv;
  const int64_t xr = DKDV ? c.p.k_rows : c.p.q_rows, yr = DKDV ? c.p.q_rows : c.p.k_rows;
  const int xh = DKDV ? c.p.kv_heads : c.p.heads, yh = DKDV ? c.p.heads : c.p.kv_heads;
  if (!encode_heads(&m.x1, x1, xr, xh, c.p.d, lx1, RT) || !encode_heads(&m.x2, x2, xr, xh, c.p.d, lx2, RT)) return cudaErrorInvalidValue;
  if (yr > 0) {
    if (!encode_heads(&m.y1, y1, yr, yh, c.p.d, ly1, CT) || !encode_heads(&m.y2, y2, yr, yh, c.p.d, ly2, CT)) return cudaErrorInvalidValue;
  } else {
    m.y1 = m.y2 = m.x1;
  }
  if (DKDV) m.x3 = m.x1;
  else if (!encode_heads(&m.x3, c.out, xr, xh, c.p.d, c.ldo, RT)) return cudaErrorInvalidValue;
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_backward_tc_kernel<SLABS, DKDV, XT>, (int)L::BYTES)) return e;
  const int sms = current_device_sm_count();
  if (sms < 1) return cudaErrorInvalidDevice;
  const int tiles = ((DKDV ? c.p.max_k : c.p.max_q) + RT - 1) / RT, total = c.p.sequences * xh * tiles;
  packed_backward_tc_kernel<SLABS, DKDV, XT><<<total < sms ? total : sms, TC_THREADS, L::BYTES, s>>>(m, c, total, tiles);
  return cudaGetLastError();
}

}  // namespace

// Columns of tensor memory decide where a piece's rows are held: 2 x 64 + d + d / 2 of a warpgroup's 256 in
// the forward pass, 256 + 2 d + d of 512 for dk and dv, 256 + d + d for dq.
cudaError_t launch_attention_packed_bf16(const PackedCall& c, cudaStream_t s) {
  if (c.p.d <= 64) return launch_forward<1, true>(c, s);
  return c.p.d <= 80 ? launch_forward<2, true>(c, s) : launch_forward<2, false>(c, s);
}
cudaError_t launch_attention_packed_dkdv_bf16(const PackedCall& c, cudaStream_t s) {
  if (c.p.d <= 64) return launch_backward<1, true, true>(c, s);
  return c.p.d <= 80 ? launch_backward<2, true, true>(c, s) : launch_backward<2, true, false>(c, s);
}
cudaError_t launch_attention_packed_dq_bf16(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 64 ? launch_backward<1, false, true>(c, s) : launch_backward<2, false, true>(c, s);
}

}  // namespace vit
