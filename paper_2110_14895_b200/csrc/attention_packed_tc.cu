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
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;
constexpr long long DRAIN_LIMIT_CYCLES = 1ll << 24;    // teardown after a failed wait: ~10 ms

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
__device__ __forceinline__ bool warp_wait(uint32_t bar, int parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, (uint32_t)parity, abort_flag));
}
// the same without letting the hardware suspend the warp: for the one warp that issues the products, which
// otherwise takes a few hundred cycles to come back
__device__ __forceinline__ bool warp_spin(uint32_t bar, int parity, volatile int* abort_flag) {
  const long long t0 = clock64();
  for (;;) {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(done) : "r"(bar), "r"((uint32_t)parity) : "memory");
    if (__all_sync(0xffffffffu, done)) return true;
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

// S[128 x n] = X[128 rows] . Y[n rows]^T over the head's channels, both operands as slabs of 64 channels
template <int SLABS, int X_ROWS, int Y_ROWS>
__device__ __forceinline__ void issue_scores(uint32_t d_tmem, uint32_t x, uint32_t y, int n, int ksteps) {
  const uint32_t id = idesc(n, false);
  const uint64_t xd = desc_sw128(x), yd = desc_sw128(y);
#pragma unroll
  for (int k = 0; k < 4 * SLABS; ++k)
    if (k < ksteps)
      umma_bf16(d_tmem, xd + (uint64_t)((k >> 2) * (X_ROWS * 8) + 2 * (k & 3)), yd + (uint64_t)((k >> 2) * (Y_ROWS * 8) + 2 * (k & 3)), id,
                k > 0 ? 1u : 0u);
}
// D[128 x d] (+)= P[128 x 16 ksteps] . Y[16 ksteps rows x d], P packed in tensor memory
template <int Y_ROWS>
__device__ __forceinline__ void issue_weighted(uint32_t d_tmem, uint32_t p_tmem, uint32_t y, int d, int ksteps, bool first) {
  const uint32_t id = idesc(d, true);
  const uint64_t yd = desc_sw128(y, Y_ROWS * 128);
#pragma unroll
  for (int k = 0; k < Y_ROWS / 16; ++k)
    if (k < ksteps) umma_bf16_ts(d_tmem, p_tmem + (uint32_t)(8 * k), yd + (uint64_t)(k * 128), id, first && k == 0 ? 0u : 1u);
}

// ============================================================================================ forward
// One block per (sequence, head, 128 queries): warps 0-3 softmax, warp 4 MMA, warp 5 TMA.  Two blocks share
// an SM (256 columns of tensor memory each): while one is in its exp2 phase the tensor core works for the
// other.  Keys come in tiles of 128.  The accumulator is rescaled only when a row's maximum has grown by
// more than 2^8 since the last time (probabilities stay below 2^8, the row sum in fp32).
struct ForwardMaps { CUtensorMap q, k, v; };

template <int SLABS>
struct ForwardSmem {
  static constexpr int STAGES = SLABS == 1 ? 2 : 1;
  static constexpr uint32_t TILE = SLABS * RT * 128;
  static constexpr uint32_t OFF_K = TILE, OFF_V = OFF_K + STAGES * TILE, OFF_BARS = OFF_V + STAGES * TILE;
  static constexpr uint32_t BYTES = OFF_BARS + 256 + 1024;
};
constexpr int FWD_THREADS = 192;
constexpr uint32_t FWD_TMEM = 256, O_COL = 128;
enum FwdBar : int { F_Q = 0, F_KFULL, F_KFREE = F_KFULL + 2, F_VFULL = F_KFREE + 2, F_VFREE = F_VFULL + 2, F_S = F_VFREE + 2, F_P, F_O, F_DRAIN, F_BARS };

template <int SLABS>
__global__ void __launch_bounds__(FWD_THREADS, 2)
packed_forward_tc_kernel(const __grid_constant__ ForwardMaps maps, const PackedCall c) {
  using L = ForwardSmem<SLABS>;
  extern __shared__ uint8_t smem_raw[];
  const int tiles = (c.p.max_q + RT - 1) / RT;
  const int tile = blockIdx.x % tiles, head = blockIdx.x / tiles % c.p.heads, seq = blockIdx.x / tiles / c.p.heads;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status)) return;
  const int q0 = tile * RT;
  if (q0 >= r.q_len) return;
  const int d = c.p.d, kv = head / (c.p.heads / c.p.kv_heads);
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int row = q0 + (warp & 3) * 32 + lane;                   // softmax warps: this thread's query
  const int64_t at = (int64_t)r.q_begin + row;
  const int n_tiles = (r.k_len + RT - 1) / RT;
  if (n_tiles == 0) {                                            // no keys
    if (warp < 4 && row < r.q_len) {
      bf16* out = static_cast<bf16*>(c.out) + at * c.ldo + (int64_t)head * d;
      for (int i = 0; i < d; i += 8) *reinterpret_cast<uint4*>(out + i) = make_uint4(0u, 0u, 0u, 0u);
      c.lse[(int64_t)head * c.p.q_rows + at] = -INFINITY;
    }
    return;
  }
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sb = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BARS);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(&bars[F_BARS]);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < F_BARS; ++i) mbar_init(bar(i), i == F_P ? 4 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 4) tmem_alloc(smem_u32(tmem_slot), FWD_TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);

  if (warp == 5) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      mbar_arrive_expect_tx(bar(F_Q), L::TILE);
      for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + s * RT * 128, &maps.q, 64 * s, head, r.q_begin + q0, bar(F_Q));
      int armed = 0;
      bool ok = true;
      for (int j = 0; j < n_tiles && ok; ++j) {
        const int st = j % L::STAGES, ph = (j / L::STAGES) & 1;
        const int krow = r.k_begin + j * RT;
        if (!mbar_wait(bar(F_KFREE + st), ph ^ 1, abort_flag)) { ok = false; break; }
        mbar_arrive_expect_tx(bar(F_KFULL + st), L::TILE);
        for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + L::OFF_K + st * L::TILE + s * RT * 128, &maps.k, 64 * s, kv, krow, bar(F_KFULL + st));
        armed = 2 * j + 1;
        if (!mbar_wait(bar(F_VFREE + st), ph ^ 1, abort_flag)) { ok = false; break; }
        mbar_arrive_expect_tx(bar(F_VFULL + st), L::TILE);
        for (int s = 0; s < SLABS; ++s) tma_load_3d(sb + L::OFF_V + st * L::TILE + s * RT * 128, &maps.v, 64 * s, kv, krow, bar(F_VFULL + st));
        armed = 2 * j + 2;
      }
      if (*abort_flag) {
        // a wait gave up somewhere: let the copies that were started land before the block leaves
        volatile int never = 0;
        mbar_wait_limit(bar(F_Q), 0, &never, DRAIN_LIMIT_CYCLES);
        for (int i = armed > 2 * L::STAGES ? armed - 2 * L::STAGES : 0; i < armed; ++i) {
          const int j = i >> 1, st = j % L::STAGES;
          mbar_wait_limit(bar((i & 1 ? F_VFULL : F_KFULL) + st), (j / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
        }
      }
    }
  } else if (warp == 4) {
    // ------------------------------------------------------------------ MMA issuer (the whole warp keeps step)
    bool ok = warp_spin(bar(F_Q), 0, abort_flag);
    for (int j = 0; j < n_tiles && ok; ++j) {
      const int st = j % L::STAGES, ph = (j / L::STAGES) & 1;
      const int here = min(RT, r.k_len - j * RT), n16 = (here + 15) / 16;
      const uint32_t ks = sb + L::OFF_K + st * L::TILE, vs = sb + L::OFF_V + st * L::TILE;
      if (!warp_spin(bar(F_KFULL + st), ph, abort_flag)) { ok = false; break; }
      __syncwarp();
      if (elect_one()) {
        // the scores overwrite P of tile j - 1: its product was issued before, by this thread
        issue_scores<SLABS, RT, RT>(tmem, sb, ks, 16 * n16, d / 16);
        umma_commit(bar(F_S));
        umma_commit(bar(F_KFREE + st));
      }
      __syncwarp();                                            // lanes that poll would hold up the one that issues
      if (!warp_spin(bar(F_VFULL + st), ph, abort_flag)) { ok = false; break; }
      __syncwarp();
      // rows of V behind the last key meet probabilities of zero: make them zero too, whatever lies there
      if (here < 16 * n16) zero_rows(vs, RT, SLABS, here, lane);
      if (!warp_spin(bar(F_P), j & 1, abort_flag)) { ok = false; break; }
      __syncwarp();
      if (elect_one()) {
        tc_fence_after();
        issue_weighted<RT>(tmem + O_COL, tmem, vs, d, n16, j == 0);
        umma_commit(bar(F_VFREE + st));
        if (j == n_tiles - 1) umma_commit(bar(F_O));
      }
      __syncwarp();
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      volatile int never = 0;
      umma_commit(bar(F_DRAIN));
      mbar_wait_limit(bar(F_DRAIN), 0, &never, DRAIN_LIMIT_CYCLES);
    }
  } else {
    // ------------------------------------------------------------------ softmax and epilogue
    const uint32_t taddr = tmem + ((uint32_t)(warp * 32) << 16);
    const float sl2 = c.p.scale * LOG2E;
    const bool warp_active = q0 + warp * 32 < r.q_len;
    float m = -INFINITY, l = 0.f;                       // row maximum in use (raw scores), row sum
    bool ok = true;
    for (int j = 0; j < n_tiles && ok; ++j) {
      const int here = min(RT, r.k_len - j * RT);
      const int nch = (here + 31) / 32;
      if (!warp_wait(bar(F_S), j & 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      if (warp_active) {
        uint32_t x[2][32];
        float top = -INFINITY;
        // pass 1: row maximum
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          if (i >= nch) break;
          tmem_ld32(taddr + (uint32_t)(32 * i), x[0]);
          tmem_ld32(taddr + (uint32_t)(32 * (i + 1)), x[1]);
          tmem_ld_wait_for(x[0]);
          tmem_ld_wait_for(x[1]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int left = here - 32 * (i + h);
            if (left >= 32) {
              float m2[2] = {top, top};
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                asm("max.f32 %0, %0, %1, %2;" : "+f"(m2[0]) : "f"(__uint_as_float(x[h][e])), "f"(__uint_as_float(x[h][e + 1])));
                asm("max.f32 %0, %0, %1, %2;" : "+f"(m2[1]) : "f"(__uint_as_float(x[h][e + 2])), "f"(__uint_as_float(x[h][e + 3])));
              }
              top = fmaxf(m2[0], m2[1]);
            } else {
#pragma unroll
              for (int e = 0; e < 32; ++e)
                if (e < left) top = fmaxf(top, __uint_as_float(x[h][e]));
            }
          }
        }
        const bool grow = (top - m) * sl2 > 8.f;         // false for NaN and for -infinity over -infinity
        if (__any_sync(0xffffffffu, grow)) {
          const float factor = grow ? (m == -INFINITY ? 0.f : ex2_approx((m - top) * sl2)) : 1.f;
          if (grow) m = top;
          l *= factor;
          if (j > 0) {                                   // the products of tile j - 1 are complete: this tile's scores are
            for (int g = 0; g < d / 16; ++g) {
              uint32_t o[16];
              tmem_ld16(taddr + O_COL + (uint32_t)(16 * g), o);
              tmem_ld_wait();
#pragma unroll
              for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * factor);
              tmem_st16(taddr + O_COL + (uint32_t)(16 * g), o);
            }
          }
        }
        // pass 2: p = exp2((s - m) sl2), row sum, P (bf16 pairs) over columns this thread has read
        const float nm = m == -INFINITY ? 0.f : -m * sl2;
        const float2 sl2v = make_float2(sl2, sl2), nmv = make_float2(nm, nm);
        float2 l2 = make_float2(0.f, 0.f);
        tmem_ld32(taddr, x[0]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= nch) break;
          tmem_ld_wait_for(x[i & 1]);
          if (i + 1 < 4 && i + 1 < nch) tmem_ld32(taddr + (uint32_t)(32 * (i + 1)), x[(i + 1) & 1]);
          const uint32_t (&s)[32] = x[i & 1];
          uint32_t pk[16];
          const int left = here - 32 * i;
          if (left >= 32) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float2 y = __ffma2_rn(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), sl2v, nmv);
              const float2 p = make_float2(ex2_approx(y.x), ex2_approx(y.y));
              l2 = __fadd2_rn(l2, p);
              pk[e] = pack_bf16(p.x, p.y);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float p0 = 2 * e < left ? ex2_approx(fmaf(__uint_as_float(s[2 * e]), sl2, nm)) : 0.f;
              const float p1 = 2 * e + 1 < left ? ex2_approx(fmaf(__uint_as_float(s[2 * e + 1]), sl2, nm)) : 0.f;
              l2.x += p0;
              l2.y += p1;
              pk[e] = pack_bf16(p0, p1);
            }
          }
          tmem_st16(taddr + (uint32_t)(16 * i), pk);
        }
        l += l2.x + l2.y;
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(F_P));
    }
    if (ok && warp_wait(bar(F_O), 0, abort_flag)) {
      tc_fence_after();
      if (warp_active) {
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        bf16* out = static_cast<bf16*>(c.out) + at * c.ldo + (int64_t)head * d;
        for (int g = 0; g < d / 16; ++g) {
          uint32_t o[16];
          tmem_ld16(taddr + O_COL + (uint32_t)(16 * g), o);
          tmem_ld_wait();
          if (row < r.q_len) store_16_bf16(out + 16 * g, o, inv);
        }
        if (row < r.q_len) c.lse[(int64_t)head * c.p.q_rows + at] = l == 0.f ? -INFINITY : fmaf(m, c.p.scale, log2f(l) * LN2);
      }
    }
  }
  // ---------------------------------------------------------------------- teardown
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (threadIdx.x == 0 && *abort_flag) atomicExch(c.dev_status, (int)VIT_ERR_TIMEOUT);
  if (warp == 4) {
    __syncwarp();
    tmem_dealloc(tmem, FWD_TMEM);
  }
}

// ============================================================================================ backward
// Two kernels of one form.  A block keeps a tile of 128 rows X1, X2 and walks over tiles of 64 rows Y1, Y2:
//   S = X1 Y1^T, dP = X2 Y2^T;  P = exp2(S sl2 - lse2), dS = P (dP - delta)
//   DKDV: X = K, V; Y = Q, dout of every query head that shares the key head (scores transposed);
//         dv += P Y2, dk += dS Y1
//   DQ:   X = Q, dout; Y = K, V;  dq += dS Y1
// NB warpgroups take the tiles in turn, each with its own columns of tensor memory for S and dP, so that
// the tensor core works for one while the others are in their exp2 phase; the MMA warp runs NB - 1 tiles ahead.
struct BackwardMaps { CUtensorMap x1, x2, y1, y2; };

constexpr int CT = 64;                                 // rows of a Y tile = columns of a tile of scores
template <int SLABS, bool DKDV, int NB>
struct BackwardCfg {
  static constexpr int STAGES = NB + 2;
  static constexpr int THREADS = NB * 128 + 64;
  static constexpr uint32_t XTILE = SLABS * RT * 128, YTILE = SLABS * CT * 128;
  static constexpr uint32_t OFF_Y = 2 * XTILE, OFF_COL = OFF_Y + STAGES * 2 * YTILE;   // float2 [STAGES][64]: -lse2, -delta of the columns
  static constexpr uint32_t OFF_BARS = OFF_COL + STAGES * CT * 8;
  static constexpr uint32_t BYTES = OFF_BARS + 512 + 1024;
  static constexpr uint32_t ACC = 64 * SLABS;          // columns of one accumulator
  static constexpr uint32_t USED = NB * 2 * CT + (DKDV ? 2 : 1) * ACC;
  static constexpr uint32_t TMEM = USED <= 256 ? 256 : 512;
  static constexpr uint32_t ACC1 = NB * 2 * CT, ACC2 = ACC1 + (DKDV ? ACC : 0);        // dv; dk or dq
  static_assert(USED <= 512 && BYTES <= 227 * 1024, "fits an SM");
};
enum BwdBar : int { B_X = 0, B_FULL, B_FREE = B_FULL + 5, B_S = B_FREE + 5, B_P = B_S + 4, B_ACC = B_P + 4, B_DRAIN, B_BARS };

template <int SLABS, bool DKDV, int NB>
__global__ void __launch_bounds__(NB * 128 + 64, NB == 1 ? 2 : 1)
packed_backward_tc_kernel(const __grid_constant__ BackwardMaps maps, const PackedCall c) {
  using L = BackwardCfg<SLABS, DKDV, NB>;
  extern __shared__ uint8_t smem_raw[];
  const int max_x = DKDV ? c.p.max_k : c.p.max_q, x_heads = DKDV ? c.p.kv_heads : c.p.heads;
  const int tiles = (max_x + RT - 1) / RT;
  const int tile = blockIdx.x % tiles, xh = blockIdx.x / tiles % x_heads, seq = blockIdx.x / tiles / x_heads;
  SeqRange r;
  if (!seq_range(c.p, seq, r, c.dev_status)) return;
  const int x_begin = DKDV ? r.k_begin : r.q_begin, x_len = DKDV ? r.k_len : r.q_len;
  const int y_begin = DKDV ? r.q_begin : r.k_begin, y_len = DKDV ? r.q_len : r.k_len;
  const int x0 = tile * RT;
  if (x0 >= x_len) return;
  const int d = c.p.d, group = c.p.heads / c.p.kv_heads;
  const int warp = (int)uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
  const int y_tiles = (y_len + CT - 1) / CT;
  const int n = DKDV ? group * y_tiles : y_tiles;      // tiles in all, head after head
  const int row = x0 + (warp & 3) * 32 + lane;         // score warps: this thread's row of X
  const int64_t at = (int64_t)x_begin + row;
  bf16* g1 = DKDV ? static_cast<bf16*>(c.dv) + at * c.lddv + (int64_t)xh * d : nullptr;
  bf16* g2 = DKDV ? static_cast<bf16*>(c.dk) + at * c.lddk + (int64_t)xh * d : static_cast<bf16*>(c.dq) + at * c.lddq + (int64_t)xh * d;
  if (n == 0) {                                        // nothing attends or is attended to: zero
    if (warp < 4 && row < x_len)
      for (int i = 0; i < d; i += 8) {
        *reinterpret_cast<uint4*>(g2 + i) = make_uint4(0u, 0u, 0u, 0u);
        if (DKDV) *reinterpret_cast<uint4*>(g1 + i) = make_uint4(0u, 0u, 0u, 0u);
      }
    return;
  }
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  const uint32_t sb = smem_u32(smem);
  uint64_t* bars = reinterpret_cast<uint64_t*>(smem + L::OFF_BARS);
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(&bars[B_BARS]);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  constexpr int MMA_WARP = NB * 4, TMA_WARP = MMA_WARP + 1;
  if (threadIdx.x == 0) {
    *abort_flag = 0;
    for (int i = 0; i < B_BARS; ++i) mbar_init(bar(i), i >= B_P && i < B_P + 4 ? 4 : 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == MMA_WARP) tmem_alloc(smem_u32(tmem_slot), L::TMEM);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(*tmem_slot);

  if (warp == TMA_WARP) {
    // ------------------------------------------------------------------ producer (the whole warp keeps step)
    if (lane == 0) {
      mbar_arrive_expect_tx(bar(B_X), 2 * L::XTILE);
      for (int s = 0; s < SLABS; ++s) {
        tma_load_3d(sb + s * RT * 128, &maps.x1, 64 * s, xh, x_begin + x0, bar(B_X));
        tma_load_3d(sb + L::XTILE + s * RT * 128, &maps.x2, 64 * s, xh, x_begin + x0, bar(B_X));
      }
    }
    int armed = 0;
    for (int t = 0; t < n; ++t) {
      const int st = t % L::STAGES, ph = (t / L::STAGES) & 1;
      const int yh = DKDV ? xh * group + t / y_tiles : xh / group;
      const int y0 = (DKDV ? t % y_tiles : t) * CT;
      const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE;
      // DKDV: the numbers of the tile's columns travel with it, negated; beyond the sequence
      // P = exp2(0 - infinity) = 0 and dS = 0.  They are in flight while this warp waits for the stage.
      float2 v[2];
      if (DKDV) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          v[i] = make_float2(INFINITY, 0.f);
          if (y0 + 32 * i + lane < y_len) v[i] = c.delta[(int64_t)yh * c.p.q_rows + y_begin + y0 + 32 * i + lane];
        }
      }
      if (!warp_wait(bar(B_FREE + st), ph ^ 1, abort_flag)) break;
      if (DKDV) {
        float2* col = reinterpret_cast<float2*>(smem + L::OFF_COL) + st * CT;
#pragma unroll
        for (int i = 0; i < 2; ++i) col[32 * i + lane] = make_float2(-v[i].x, -v[i].y);
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
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      // a wait gave up somewhere: let the copies that were started land before the block leaves
      volatile int never = 0;
      mbar_wait_limit(bar(B_X), 0, &never, DRAIN_LIMIT_CYCLES);
      for (int t = armed > L::STAGES ? armed - L::STAGES : 0; t < armed; ++t)
        mbar_wait_limit(bar(B_FULL + t % L::STAGES), (t / L::STAGES) & 1, &never, DRAIN_LIMIT_CYCLES);
    }
  } else if (warp == MMA_WARP) {
    // ------------------------------------------------------------------ MMA issuer (the whole warp keeps step)
    bool ok = warp_spin(bar(B_X), 0, abort_flag);
    for (int t = 0; t < n + NB - 1 && ok; ++t) {
      if (t < n) {
        const int st = t % L::STAGES, b = t % NB;
        const int here = min(CT, y_len - (DKDV ? t % y_tiles : t) * CT), n16 = (here + 15) / 16;
        const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE;
        if (!warp_spin(bar(B_FULL + st), (t / L::STAGES) & 1, abort_flag)) { ok = false; break; }
        __syncwarp();
        // rows of Y behind the end of the sequence become zero, whatever lies there: they meet weights of
        // zero in the second products, and give scores of zero in the first
        if (here < 16 * n16) {
          zero_rows(y, CT, SLABS, here, lane);
          zero_rows(y + L::YTILE, CT, SLABS, here, lane);
        }
        if (elect_one()) {
          // S and dP overwrite P and dS of tile t - NB: their products were issued before, by this thread
          const uint32_t s_col = tmem + (uint32_t)(b * 2 * CT);
          issue_scores<SLABS, RT, CT>(s_col, sb, y, 16 * n16, d / 16);
          issue_scores<SLABS, RT, CT>(s_col + CT, sb + L::XTILE, y + L::YTILE, 16 * n16, d / 16);
          umma_commit(bar(B_S + b));
        }
        __syncwarp();                                          // lanes that poll would hold up the one that issues
      }
      const int u = t - (NB - 1);
      if (u >= 0) {
        const int st = u % L::STAGES, b = u % NB;
        const int here = min(CT, y_len - (DKDV ? u % y_tiles : u) * CT), n16 = (here + 15) / 16;
        const uint32_t y = sb + L::OFF_Y + st * 2 * L::YTILE, s_col = tmem + (uint32_t)(b * 2 * CT);
        if (!warp_spin(bar(B_P + b), (u / NB) & 1, abort_flag)) { ok = false; break; }
        __syncwarp();
        if (elect_one()) {
          tc_fence_after();
          if (DKDV) issue_weighted<CT>(tmem + L::ACC1, s_col, y + L::YTILE, d, n16, u == 0);
          issue_weighted<CT>(tmem + L::ACC2, s_col + CT, y, d, n16, u == 0);
          umma_commit(bar(B_FREE + st));
          if (u == n - 1) umma_commit(bar(B_ACC));
        }
        __syncwarp();
      }
    }
    __syncwarp();
    if (*abort_flag && lane == 0) {
      volatile int never = 0;
      umma_commit(bar(B_DRAIN));
      mbar_wait_limit(bar(B_DRAIN), 0, &never, DRAIN_LIMIT_CYCLES);
    }
  } else {
    // ------------------------------------------------------------------ probabilities and their gradients
    const int wg = warp >> 2;
    const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
    const uint32_t taddr = lanes + (uint32_t)(wg * 2 * CT);
    const float sl2 = c.p.scale * LOG2E;
    const float2 sl2v = make_float2(sl2, sl2);
    const bool warp_active = x0 + (warp & 3) * 32 < x_len;
    float2 mine = make_float2(0.f, 0.f);                 // DQ: of this thread's row
    if (!DKDV && row < x_len) mine = c.delta[(int64_t)xh * c.p.q_rows + at];
    const float2 nls = make_float2(-mine.x, -mine.x), nde = make_float2(-mine.y, -mine.y);
    bool ok = true;
    for (int t = wg; t < n && ok; t += NB) {
      const int here = min(CT, y_len - (DKDV ? t % y_tiles : t) * CT), nch = (here + 31) / 32;
      const int st = t % L::STAGES;
      const float4* col = reinterpret_cast<const float4*>(smem + L::OFF_COL) + st * (CT / 2);   // two columns each
      if (DKDV && !warp_wait(bar(B_FULL + st), (t / L::STAGES) & 1, abort_flag)) { ok = false; break; }
      if (!warp_wait(bar(B_S + wg), (t / NB) & 1, abort_flag)) { ok = false; break; }
      tc_fence_after();
      if (warp_active) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (i >= nch) break;
          uint32_t s[32], g[32];
          tmem_ld32(taddr + (uint32_t)(32 * i), s);
          tmem_ld32(taddr + (uint32_t)(CT + 32 * i), g);
          tmem_ld_wait_for(s);
          tmem_ld_wait_for(g);
          uint32_t pk[16], dk[16];
          const int left = here - 32 * i;
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            float2 a = nls, b = nde;
            if (DKDV) {
              const float4 v = col[16 * i + e];
              a = make_float2(v.x, v.z);
              b = make_float2(v.y, v.w);
            }
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(s[2 * e]), __uint_as_float(s[2 * e + 1])), sl2v, a);
            float2 p = make_float2(ex2_approx(x.x), ex2_approx(x.y));
            if (!DKDV && left < 32) {                      // keys behind the end
              if (2 * e >= left) p.x = 0.f;
              if (2 * e + 1 >= left) p.y = 0.f;
            }
            const float2 y = __fmul2_rn(p, __fadd2_rn(make_float2(__uint_as_float(g[2 * e]), __uint_as_float(g[2 * e + 1])), b));
            if (DKDV) pk[e] = pack_bf16(p.x, p.y);
            dk[e] = pack_bf16(y.x, y.y);
          }
          if (DKDV) tmem_st16(taddr + (uint32_t)(16 * i), pk);
          tmem_st16(taddr + (uint32_t)(CT + 16 * i), dk);
        }
        tmem_st_wait();
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(B_P + wg));
    }
    if (ok && warp_wait(bar(B_ACC), 0, abort_flag)) {
      tc_fence_after();
      if (warp_active) {
        for (int i = wg; i < d / 16 * (DKDV ? 2 : 1); i += NB) {
          const bool second = i >= d / 16;
          const int cc = 16 * (second ? i - d / 16 : i);
          uint32_t o[16];
          tmem_ld16(lanes + (second ? L::ACC1 : L::ACC2) + (uint32_t)cc, o);
          tmem_ld_wait();
          if (row < x_len) store_16_bf16((second ? g1 : g2) + cc, o, second ? 1.f : c.p.scale);
        }
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
    tmem_dealloc(tmem, L::TMEM);
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

template <int SLABS>
cudaError_t launch_forward(const PackedCall& c, cudaStream_t s) {
  using L = ForwardSmem<SLABS>;
  ForwardMaps m;
  if (!encode_heads(&m.q, c.q, c.p.q_rows, c.p.heads, c.p.d, c.ldq, RT)) return cudaErrorInvalidValue;
  if (c.p.k_rows > 0) {
    if (!encode_heads(&m.k, c.k, c.p.k_rows, c.p.kv_heads, c.p.d, c.ldk, RT)) return cudaErrorInvalidValue;
    if (!encode_heads(&m.v, c.v, c.p.k_rows, c.p.kv_heads, c.p.d, c.ldv, RT)) return cudaErrorInvalidValue;
  } else {
    m.k = m.v = m.q;                                   // no keys at all: never used
  }
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_forward_tc_kernel<SLABS>, (int)L::BYTES)) return e;
  const int tiles = (c.p.max_q + RT - 1) / RT;
  packed_forward_tc_kernel<SLABS><<<c.p.sequences * c.p.heads * tiles, FWD_THREADS, L::BYTES, s>>>(m, c);
  return cudaGetLastError();
}

template <int SLABS, bool DKDV, int NB>
cudaError_t launch_backward(const PackedCall& c, cudaStream_t s) {
  using L = BackwardCfg<SLABS, DKDV, NB>;
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
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, packed_backward_tc_kernel<SLABS, DKDV, NB>, (int)L::BYTES)) return e;
  const int tiles = ((DKDV ? c.p.max_k : c.p.max_q) + RT - 1) / RT;
  packed_backward_tc_kernel<SLABS, DKDV, NB><<<c.p.sequences * xh * tiles, L::THREADS, L::BYTES, s>>>(m, c);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_attention_packed_bf16(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 64 ? launch_forward<1>(c, s) : launch_forward<2>(c, s);
}
cudaError_t launch_attention_packed_dkdv_bf16(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 64 ? launch_backward<1, true, 1>(c, s) : launch_backward<2, true, 2>(c, s);
}
cudaError_t launch_attention_packed_dq_bf16(const PackedCall& c, cudaStream_t s) {
  return c.p.d <= 64 ? launch_backward<1, false, 1>(c, s) : launch_backward<2, false, 2>(c, s);
}

}  // namespace vit
