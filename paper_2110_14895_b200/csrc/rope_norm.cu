// Rotary positions on several axes, alone or behind the root-mean-square norm of every query and
// key head, and the gradients of the latter.
//
//   y = R x                                  pair i of a head turned by positions[axis(i)][row] * freqs[i]
//   y = R (g x / sqrt(mean(x^2) + eps))      norm, gain, rotation
//   u = R^T dy, xh = x rstd, w = g u:        dx = rstd (w - xh mean(w xh)),  dg = sum over rows and heads of u xh
//
// All of them are bound by HBM: every element is read once and written once, in 16-byte pieces.  A warp takes a
// row (or an equal part of its heads) at a time; a head belongs to d / 8 neighbouring lanes, eight channels to a
// lane, as many heads side by side as fit (d = 80: three heads on 30 lanes), so that the sums of the norm are a
// few shuffles and nothing of a head leaves its warp.  The angles of a row are shared by its heads: the warp
// turns them into cosines and sines once, in shared memory of its own, while its first heads are on their way,
// and every lane keeps those of its eight channels in registers.  Warps never wait for one another.
#include "vit_internal.h"
#include "sm100_ptx.cuh"
#include "lane_groups.cuh"

#include <cmath>

namespace vit {

namespace {

constexpr int WARPS = 4, THREADS = 32 * WARPS;
constexpr int CH = 8;                       // channels of a lane
constexpr int MAX_SMS = 256;
constexpr int MAX_PAIRS = 64;               // of a head

// A row's cosines and sines, one table to a warp; read in pieces of two pairs
struct alignas(16) TurnTable { float2 of[MAX_PAIRS]; };
static_assert(alignof(TurnTable) >= alignof(float4) && sizeof(TurnTable) % alignof(float4) == 0, "every warp's table can be read as float4");

enum Rotation { INTERLEAVED = 0, HALVES_BY_LANES = 1, HALVES_ANY = 2 };
enum Mode { TURN = 0, NORM_TURN = 1, NORM_TURN_GRAD = 2 };

struct RopeNormArgs {
  int rows, heads, q_heads, d;
  int lanes, side;                          // lanes of a head (d / 8), heads side by side in a warp
  int n_pairs, first_pair[5];               // axis a turns the pairs [first_pair[a], first_pair[a + 1])
  int split;                                // warps that share a row's heads
  float turn_sign;                          // +1: by the angle, -1: back
  float eps, inv_d;
  const int32_t* positions;                 // [axes][rows]
  const float* freqs;                       // [n_pairs]
  const float *q_gain, *k_gain;             // [d]
  const void* x;  int64_t ldx;
  const void* dy; int64_t lddy;             // NORM_TURN_GRAD
  void* y;        int64_t ldy;              // y, or dx
  float* partial;                           // NORM_TURN_GRAD: [gridDim.x][2][d]
  int stages;                               // rows of a warp's ring in shared memory
  int* dev_status;
};

template <typename T> struct Piece;         // eight channels as they lie in memory
template <> struct Piece<bf16> { uint4 v; };
template <> struct Piece<float> { float4 v[2]; };

__device__ __forceinline__ void load_piece(Piece<bf16>& p, const bf16* a) { p.v = *reinterpret_cast<const uint4*>(a); }
__device__ __forceinline__ void load_piece(Piece<float>& p, const float* a) {
  p.v[0] = reinterpret_cast<const float4*>(a)[0];
  p.v[1] = reinterpret_cast<const float4*>(a)[1];
}
__device__ __forceinline__ void unpack(const Piece<bf16>& p, float (&f)[CH]) {
  const uint32_t w[4] = {p.v.x, p.v.y, p.v.z, p.v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack(const Piece<float>& p, float (&f)[CH]) {
  f[0] = p.v[0].x; f[1] = p.v[0].y; f[2] = p.v[0].z; f[3] = p.v[0].w;
  f[4] = p.v[1].x; f[5] = p.v[1].y; f[6] = p.v[1].z; f[7] = p.v[1].w;
}
__device__ __forceinline__ void store_piece(bf16* a, const float (&f)[CH]) {   // the one rounding to bf16
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(a) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store_piece(float* a, const float (&f)[CH]) {
  reinterpret_cast<float4*>(a)[0] = make_float4(f[0], f[1], f[2], f[3]);
  reinterpret_cast<float4*>(a)[1] = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void load_floats(float (&f)[CH], const float* a) {
  Piece<float> p;
  load_piece(p, a);
  unpack(p, f);
}
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(float v) { return v; }

// Cosine and sine of position * freq.  The product of a 31-bit position and a 24-bit frequency has 55 bits, two more
// than a double: product and turns are taken in two parts each, so that the part of a turn that is left is good to
// 32 bits for angles up to 2^52 (one part alone is off by |angle| 2^-52: 4e-7 at 2^31, 0.3 at 2^31 times a frequency
// of 10^6).  __dmul_rn: the products whose rounding is made up for must not become part of a sum.
__device__ __forceinline__ float2 turn_of(int32_t position, float freq) {
  constexpr double PER_TURN = 0.15915494309189533577, PER_TURN_REST = -9.839338337591243e-18;      // 1 / (2 pi)
  const double p = position, f = freq, angle = __dmul_rn(p, f), turns = __dmul_rn(angle, PER_TURN);
  const double rest = fma(angle, PER_TURN, -turns) + fma(fma(p, f, -angle), PER_TURN, angle * PER_TURN_REST);
  float s, c;
  sincospif((float)(2.0 * ((turns - rint(turns)) + rest)), &s, &c);
  return make_float2(c, s);
}

// The eight channels that are partners of a lane's eight, for the heads in flight: from the lane that has them.
__device__ __forceinline__ void fetch_partner(Piece<bf16>& to, const Piece<bf16>& p, int from) {
  to.v.x = __shfl_sync(0xffffffffu, p.v.x, from);
  to.v.y = __shfl_sync(0xffffffffu, p.v.y, from);
  to.v.z = __shfl_sync(0xffffffffu, p.v.z, from);
  to.v.w = __shfl_sync(0xffffffffu, p.v.w, from);
}
__device__ __forceinline__ void fetch_partner(Piece<float>& to, const Piece<float>& p, int from) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    to.v[i].x = __shfl_sync(0xffffffffu, p.v[i].x, from);
    to.v[i].y = __shfl_sync(0xffffffffu, p.v[i].y, from);
    to.v[i].z = __shfl_sync(0xffffffffu, p.v[i].z, from);
    to.v[i].w = __shfl_sync(0xffffffffu, p.v[i].w, from);
  }
}

// HEADS steps of a warp (of `side` heads each) are in flight at a time.
template <typename T, int ROT, int MODE, int HEADS>
__global__ void __launch_bounds__(THREADS, MODE == NORM_TURN_GRAD ? 4 : 5)
rope_norm_kernel(const RopeNormArgs p) {
  __shared__ TurnTable tables[WARPS];
  extern __shared__ float share[];                      // NORM_TURN_GRAD: [WARPS * side][2][d]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float2* table = tables[warp].of;
  const int slot = lane / p.lanes, at = lane - slot * p.lanes, first = slot * p.lanes;   // head of the step, place in it, its first lane
  const bool active = slot < p.side;
  const int c0 = at * CH, n = p.n_pairs;
  const int first_lane = active ? first : 0;

  float dq_gain[CH] = {}, dk_gain[CH] = {};             // NORM_TURN_GRAD: of this lane's channels, all rows and heads
  // out[j] = v[j] * cs[j] + partner(v)[j] * sn[j] where the channel turns
  int pair[CH];
  uint32_t turning = 0;                                 // bit j: channel j turns
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    const int c = c0 + j;
    pair[j] = ROT == INTERLEAVED ? c >> 1 : c < n ? c : c - n;
    if (active && pair[j] < n) turning |= 1u << j;
  }
  // HALVES_BY_LANES: the partner's eight channels are those of one other lane of the head
  const int partner_lane = ROT == HALVES_BY_LANES && (turning & 1) ? first + (c0 < n ? c0 + n : c0 - n) / CH : lane;
  const bool every = 2 * n == p.d;                      // no channel is passed on
  const HeadSum sums = head_sum_plan(p.lanes, at, first_lane);

  const int64_t units = (int64_t)p.rows * p.split;      // a warp's piece of work: a row, or one of `split` parts of its heads
  for (int64_t u = (int64_t)blockIdx.x * WARPS + warp; u < units; u += (int64_t)gridDim.x * WARPS) {
    const int64_t row = p.split == 1 ? u : u / p.split;
    const int part = (int)(u - row * p.split);
    const T* x = static_cast<const T*>(p.x) + row * p.ldx + c0;
    const T* dy = static_cast<const T*>(p.dy) + (MODE == NORM_TURN_GRAD ? row * p.lddy + c0 : 0);
    T* y = static_cast<T*>(p.y) + row * p.ldy + c0;
    float cs[CH], sn[CH];
    bool have_angles = false;
    // query heads, then key heads (TURN: all of them as one)
#pragma unroll 1
    for (int kind = 0; kind < (MODE == TURN ? 1 : 2); ++kind) {
      const int h_end = MODE == TURN ? p.heads : kind ? p.heads : p.q_heads;
      const int h_begin = MODE == TURN || kind == 0 ? 0 : p.q_heads;
      const int stride = p.split * p.side;              // heads of one step of all warps of the row
      const float* gains = MODE == TURN ? nullptr : kind ? p.k_gain : p.q_gain;
      float gain[CH] = {}, other_gain[CH] = {}, dg[CH] = {};   // other_gain: of the partners
      if (MODE != TURN && active) {
        load_floats(gain, gains + c0);
        if (ROT == HALVES_BY_LANES && MODE == NORM_TURN) load_floats(other_gain, gains + (partner_lane - first) * CH);
      }
#pragma unroll 1
      for (int hb = h_begin + part * p.side; hb < h_end; hb += stride * HEADS) {
        Piece<T> px[HEADS], pd[HEADS];
        bool on[HEADS];
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {               // all loads in flight before the first use
          const int h = hb + k * stride + slot;
          on[k] = active && h < h_end;
          if (on[k]) {
            load_piece(px[k], x + (int64_t)h * p.d);
            if (MODE == NORM_TURN_GRAD) load_piece(pd[k], dy + (int64_t)h * p.d);
          } else {
            px[k] = Piece<T>{};
            if (MODE == NORM_TURN_GRAD) pd[k] = Piece<T>{};
          }
        }
        if (!have_angles) {                             // of this row, while the loads are on their way
          have_angles = true;
          __syncwarp();                                 // the last row's have been read
          for (int i = lane; i < n; i += 32) {
            int axis = 0;
            while (i >= p.first_pair[axis + 1]) ++axis;
            table[i] = turn_of(p.positions[(int64_t)axis * p.rows + row], p.freqs[i]);
          }
          __syncwarp();
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            const float2 t = turning >> j & 1 ? table[pair[j]] : make_float2(1.f, 0.f);
            const bool second = ROT == INTERLEAVED ? j & 1 : c0 + j >= n;
            cs[j] = t.x;
            sn[j] = second ? p.turn_sign * t.y : -p.turn_sign * t.y;
          }
        }
#pragma unroll
        for (int k = 0; k < HEADS; ++k) {
          if (hb + k * stride >= h_end) break;          // the same for the whole warp
          const int64_t h = hb + k * stride + slot;
          float x_[CH], v[CH], o[CH], other[CH];
          unpack(px[k], x_);
          float rstd = 1.f;
          if (MODE != TURN) {
            float sq = 0.f;
#pragma unroll
            for (int j = 0; j < CH; ++j) sq = fmaf(x_[j], x_[j], sq);
            rstd = 1.0f / sqrtf(fmaf(head_sum(sq, sums), p.inv_d, p.eps));
            // a place without a head adds nothing to the gains' gradients (with eps = 0 its factor would be infinite)
            if (MODE == NORM_TURN_GRAD && !on[k]) rstd = 0.f;
          }
          // what is turned, and its partners: gradients as they come, values times gain (the norm's factor is
          // the same for the whole head and comes last)
          const Piece<T>& src = MODE == NORM_TURN_GRAD ? pd[k] : px[k];
          if (MODE == NORM_TURN_GRAD) {
            unpack(pd[k], v);
          } else {
#pragma unroll
            for (int j = 0; j < CH; ++j) v[j] = MODE == NORM_TURN ? x_[j] * gain[j] : x_[j];
          }
          if (ROT == INTERLEAVED) {
#pragma unroll
            for (int j = 0; j < CH; ++j) other[j] = v[j ^ 1];
          } else if (ROT == HALVES_BY_LANES) {
            Piece<T> pp;
            fetch_partner(pp, src, partner_lane);
            unpack(pp, other);
            if (MODE == NORM_TURN) {
#pragma unroll
              for (int j = 0; j < CH; ++j) other[j] *= other_gain[j];
            }
          } else {
            // the partner lies at any offset: read it again (it is in L1), before this head is written
#pragma unroll
            for (int j = 0; j < CH; ++j) {
              other[j] = 0.f;
              if (on[k] && (turning >> j & 1)) {
                const int c = c0 + j, q = c < n ? c + n : c - n;
                other[j] = to_f((MODE == NORM_TURN_GRAD ? dy : x)[h * p.d + q - c0]);
                if (MODE == NORM_TURN) other[j] *= gains[q];
              }
            }
          }
          if (every) {
#pragma unroll
            for (int j = 0; j < CH; ++j) o[j] = fmaf(v[j], cs[j], other[j] * sn[j]);
          } else {
            // a channel that does not turn is passed on as it is, whatever its partner holds
#pragma unroll
            for (int j = 0; j < CH; ++j) o[j] = turning >> j & 1 ? fmaf(v[j], cs[j], other[j] * sn[j]) : v[j];
          }
          if (MODE == NORM_TURN) {
#pragma unroll
            for (int j = 0; j < CH; ++j) o[j] *= rstd;
          }
          if (MODE == NORM_TURN_GRAD) {
            float dot = 0.f;
#pragma unroll
            for (int j = 0; j < CH; ++j) {
              x_[j] *= rstd;
              dg[j] = fmaf(o[j], x_[j], dg[j]);
              o[j] *= gain[j];
              dot = fmaf(o[j], x_[j], dot);
            }
            const float mean = head_sum(dot, sums) * p.inv_d;
#pragma unroll
            for (int j = 0; j < CH; ++j) o[j] = rstd * fmaf(-mean, x_[j], o[j]);
          }
          if (ROT == HALVES_ANY) __syncwarp();          // in place: every lane has read before any writes
          if (on[k]) store_piece(y + h * p.d, o);
        }
      }
      if (MODE == NORM_TURN_GRAD) {
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          if (kind) dk_gain[j] += dg[j];
          else dq_gain[j] += dg[j];
        }
      }
    }
  }

  if (MODE == NORM_TURN_GRAD) {
    // this block's share of the gains' gradients: its heads are added in a fixed order
    const int groups = WARPS * p.side;
    if (active) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        share[((warp * p.side + slot) * 2 + 0) * p.d + c0 + j] = dq_gain[j];
        share[((warp * p.side + slot) * 2 + 1) * p.d + c0 + j] = dk_gain[j];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.d; i += THREADS) {
      float sum = 0.f;
      for (int g = 0; g < groups; ++g) sum += share[g * 2 * p.d + i];
      p.partial[(int64_t)blockIdx.x * 2 * p.d + i] = sum;
    }
  }
}

// ---------------------------------------------------------------------- every channel turns (2 n = d)
// The usual case.  What bounds it besides HBM is the number of instructions (the kernel above takes 2900 for a row
// of 32 heads of 80 channels, 133 us at 32896 rows): a lane holds 16 channels of a head, both channels of its eight
// pairs among them, so that turning needs no exchange; sums run over d / 16 lanes; arithmetic is on pairs of values.
struct Sixteen { float2 a[4], b[4]; };       // HALVES: channels 8 at ..., n + 8 at ...; INTERLEAVED: 16 consecutive ones

template <typename T> struct Piece16;
template <> struct Piece16<bf16> { uint4 v[2]; };
template <> struct Piece16<float> { float4 v[4]; };
__device__ __forceinline__ void load16(Piece16<bf16>& p, const bf16* a, int second) {
  p.v[0] = *reinterpret_cast<const uint4*>(a);
  p.v[1] = *reinterpret_cast<const uint4*>(a + second);
}
__device__ __forceinline__ void load16(Piece16<float>& p, const float* a, int second) {
  p.v[0] = reinterpret_cast<const float4*>(a)[0];
  p.v[1] = reinterpret_cast<const float4*>(a)[1];
  p.v[2] = reinterpret_cast<const float4*>(a + second)[0];
  p.v[3] = reinterpret_cast<const float4*>(a + second)[1];
}
__device__ __forceinline__ void zero16(Piece16<bf16>& p) { p.v[0] = p.v[1] = make_uint4(0u, 0u, 0u, 0u); }
__device__ __forceinline__ void zero16(Piece16<float>& p) {
#pragma unroll
  for (int i = 0; i < 4; ++i) p.v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
}
__device__ __forceinline__ float2 low_high(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ void open16(const Piece16<bf16>& p, Sixteen& f) {
  f.a[0] = low_high(p.v[0].x); f.a[1] = low_high(p.v[0].y); f.a[2] = low_high(p.v[0].z); f.a[3] = low_high(p.v[0].w);
  f.b[0] = low_high(p.v[1].x); f.b[1] = low_high(p.v[1].y); f.b[2] = low_high(p.v[1].z); f.b[3] = low_high(p.v[1].w);
}
__device__ __forceinline__ void open16(const Piece16<float>& p, Sixteen& f) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    f.a[2 * i] = make_float2(p.v[i].x, p.v[i].y);
    f.a[2 * i + 1] = make_float2(p.v[i].z, p.v[i].w);
    f.b[2 * i] = make_float2(p.v[2 + i].x, p.v[2 + i].y);
    f.b[2 * i + 1] = make_float2(p.v[2 + i].z, p.v[2 + i].w);
  }
}
__device__ __forceinline__ uint32_t rounded(float2 f) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store16(bf16* a, int second, const Sixteen& f) {     // the one rounding to bf16
  *reinterpret_cast<uint4*>(a) = make_uint4(rounded(f.a[0]), rounded(f.a[1]), rounded(f.a[2]), rounded(f.a[3]));
  *reinterpret_cast<uint4*>(a + second) = make_uint4(rounded(f.b[0]), rounded(f.b[1]), rounded(f.b[2]), rounded(f.b[3]));
}
__device__ __forceinline__ void store16(float* a, int second, const Sixteen& f) {
  reinterpret_cast<float4*>(a)[0] = make_float4(f.a[0].x, f.a[0].y, f.a[1].x, f.a[1].y);
  reinterpret_cast<float4*>(a)[1] = make_float4(f.a[2].x, f.a[2].y, f.a[3].x, f.a[3].y);
  reinterpret_cast<float4*>(a + second)[0] = make_float4(f.b[0].x, f.b[0].y, f.b[1].x, f.b[1].y);
  reinterpret_cast<float4*>(a + second)[1] = make_float4(f.b[2].x, f.b[2].y, f.b[3].x, f.b[3].y);
}

__device__ __forceinline__ float2 twice(float v) { return make_float2(v, v); }

// One row to shared memory, counted on an mbarrier
__device__ __forceinline__ void copy_row(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes),
               "r"(bar)
               : "memory");
}

// RING: a warp's rows come by bulk copies into a ring of `stages` rows of its own in shared memory, so that the next
// row is on its way while one is worked on, at no cost in registers.  Without it (rows of which several warps take
// parts, or that are too long for the ring) STEPS steps of a warp (of `side` heads each) are loaded together.
// INTERLEAVED: values 2 i, 2 i + 1 of the
// sixteen are a pair; HALVES: value i of a and of b.
template <typename T, bool IL, int MODE, int STEPS, bool RING>
__global__ void __launch_bounds__(THREADS, MODE == NORM_TURN_GRAD ? 3 : 4)
rope_norm_full_kernel(const RopeNormArgs p) {
  __shared__ TurnTable tables[WARPS];
  __shared__ uint64_t bars[WARPS][4];
  __shared__ int given_up;
  extern __shared__ __align__(16) float share[];        // rings; at the end, NORM_TURN_GRAD: [WARPS * side][2][d]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float2* table = tables[warp].of;
  const int slot = lane / p.lanes, at = lane - slot * p.lanes;
  const bool active = slot < p.side;
  const int n = p.n_pairs, c0 = active ? (IL ? 16 * at : 8 * at) : 0, second = IL ? 8 : n;   // first channel of a, and of b behind it
  const HeadSum sums = head_sum_plan(p.lanes, at, active ? slot * p.lanes : 0);
  const int step = p.split * p.side;                    // heads from one step of the warp to its next
  const int64_t units = (int64_t)p.rows * p.split, next_unit = (int64_t)gridDim.x * WARPS;

  // a lane turns up to two of a row's pairs into the table; their positions are fetched a row ahead
  const int32_t* from[2];
  float freq[2] = {0.f, 0.f};
  int ahead[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    int axis = 0;
    from[e] = p.positions;
    if (lane + 32 * e < n) {
      while (lane + 32 * e >= p.first_pair[axis + 1]) ++axis;
      from[e] = p.positions + (int64_t)axis * p.rows;
      freq[e] = p.freqs[lane + 32 * e];
    }
  }
  const int64_t u0 = (int64_t)blockIdx.x * WARPS + warp;
  if (u0 < units) {
    const int64_t row = p.split == 1 ? u0 : u0 / p.split;
#pragma unroll
    for (int e = 0; e < 2; ++e) ahead[e] = from[e][row];
  }
  // the warp's ring: a stage holds a row of x, and of dy
  constexpr int KINDS = MODE == NORM_TURN_GRAD ? 2 : 1;
  const uint32_t row_bytes = (uint32_t)(p.heads * p.d) * (uint32_t)sizeof(T);
  const uint32_t ring = ptx::smem_u32(share) + (uint32_t)(warp * p.stages * KINDS) * row_bytes, bar0 = ptx::smem_u32(&bars[warp][0]);
  auto fetch_row = [&](int64_t row, int stage) {
    ptx::mbar_arrive_expect_tx(bar0 + 8 * stage, KINDS * row_bytes);
    copy_row(ring + (uint32_t)(stage * KINDS) * row_bytes, static_cast<const T*>(p.x) + row * p.ldx, row_bytes, bar0 + 8 * stage);
    if (MODE == NORM_TURN_GRAD)
      copy_row(ring + (uint32_t)(stage * KINDS + 1) * row_bytes, static_cast<const T*>(p.dy) + row * p.lddy, row_bytes, bar0 + 8 * stage);
  };
  if (RING) {
    if (threadIdx.x == 0) given_up = 0;
    if (lane == 0) {
      for (int i = 0; i < p.stages; ++i) ptx::mbar_init(bar0 + 8 * i, 1);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (lane == 0)
      for (int i = 0; i < p.stages; ++i)
        if (u0 + i * next_unit < units) fetch_row(u0 + i * next_unit, i);
  }
  int stage = 0, parity = 0;
  float2 dg[2][8];                                      // gradients of the gains: of query and of key heads
#pragma unroll
  for (int k = 0; k < 2; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) dg[k][j] = make_float2(0.f, 0.f);

#pragma unroll 1
  for (int64_t u = u0; u < units; u += next_unit) {
    const int64_t row = p.split == 1 ? u : u / p.split;
    const int first_head = ((int)(u - row * p.split)) * p.side + slot;
    const T* x = static_cast<const T*>(p.x) + row * p.ldx + c0;
    const T* dy = MODE == NORM_TURN_GRAD ? static_cast<const T*>(p.dy) + row * p.lddy + c0 : nullptr;
    T* y = static_cast<T*>(p.y) + row * p.ldy + c0;
    if (RING) {
      if (!__all_sync(0xffffffffu, ptx::mbar_wait(bar0 + 8 * stage, (uint32_t)parity, (volatile int*)&given_up))) {
        // a copy that does not come: say so, give the ones under way time to land, and leave
        volatile int never = 0;
        if (lane == 0) {
          atomicExch(p.dev_status, (int)VIT_ERR_TIMEOUT);
          for (int i = 0; i < p.stages; ++i)
            if (u + i * next_unit < units)
              ptx::mbar_wait_limit(bar0 + 8 * ((stage + i) % p.stages), (uint32_t)(parity ^ (stage + i >= p.stages)), &never, 1ll << 24);
        }
        __syncwarp();
        break;
      }
      x = reinterpret_cast<const T*>(reinterpret_cast<const char*>(share) + (size_t)(warp * p.stages + stage) * KINDS * row_bytes) + c0;
      dy = x + p.heads * p.d;
    }
    bool have_angles = false;
    Sixteen cs;                                         // of the eight pairs: a = cosines, b = sines
#pragma unroll
    for (int kind = 0; kind < (MODE == TURN ? 1 : 2); ++kind) {
      const int h_begin = kind ? p.q_heads : 0, h_end = MODE == TURN || kind ? p.heads : p.q_heads;
      Sixteen gain;
      bool have_gains = false;
#pragma unroll 1
      for (int h0 = h_begin + first_head - slot; h0 < h_end; h0 += step * STEPS) {
        Piece16<T> px[STEPS], pd[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {               // all loads in flight before the first use
          const int h = h0 + slot + k * step;
          zero16(px[k]);
          if (MODE == NORM_TURN_GRAD) zero16(pd[k]);
          if (active && h < h_end) {
            load16(px[k], x + h * p.d, second);
            if (MODE == NORM_TURN_GRAD) load16(pd[k], dy + h * p.d, second);
          }
        }
        if (!have_angles) {                             // of this row, while the loads are on their way
          have_angles = true;
          __syncwarp();                                 // the last row's have been read
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (lane + 32 * e < n) table[lane + 32 * e] = turn_of(ahead[e], freq[e]);
          __syncwarp();
          const int64_t un = u + next_unit;
          if (un < units) {
            const int64_t rn = p.split == 1 ? un : un / p.split;
#pragma unroll
            for (int e = 0; e < 2; ++e) ahead[e] = from[e][rn];
          }
          const float4* t = reinterpret_cast<const float4*>(table + 8 * at);     // (c0, s0, c1, s1)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float4 v = t[j];
            cs.a[j] = make_float2(v.x, v.z);
            cs.b[j] = make_float2(p.turn_sign * v.y, p.turn_sign * v.w);
          }
        }
        if (MODE != TURN && !have_gains) {
          have_gains = true;
          const float* g = (kind ? p.k_gain : p.q_gain) + c0;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            gain.a[j] = *reinterpret_cast<const float2*>(g + 2 * j);
            gain.b[j] = *reinterpret_cast<const float2*>(g + second + 2 * j);
          }
        }
        float rstd[STEPS];
        if (MODE != TURN) {
          // the heads' sums of squares step by step together: every step waits for a shuffle
#pragma unroll
          for (int k = 0; k < STEPS; ++k) {
            Sixteen v;
            open16(px[k], v);
            float2 sq = __fmul2_rn(v.a[0], v.a[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) sq = __ffma2_rn(v.a[j], v.a[j], sq);
#pragma unroll
            for (int j = 0; j < 4; ++j) sq = __ffma2_rn(v.b[j], v.b[j], sq);
            rstd[k] = sq.x + sq.y;
          }
          head_sums(rstd, sums);
#pragma unroll
          for (int k = 0; k < STEPS; ++k) rstd[k] = rsqrtf(fmaf(rstd[k], p.inv_d, p.eps));
        }
#pragma unroll
        for (int k = 0; k < STEPS; ++k) {
          if (h0 + k * step >= h_end) break;            // the same for the whole warp
          Sixteen v, o;
          open16(MODE == NORM_TURN_GRAD ? pd[k] : px[k], v);
          if (MODE == NORM_TURN) {
            const float2 r = twice(rstd[k]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              v.a[j] = __fmul2_rn(v.a[j], __fmul2_rn(gain.a[j], r));
              v.b[j] = __fmul2_rn(v.b[j], __fmul2_rn(gain.b[j], r));
            }
          }
          if (IL) {
            // pair q is v.a[q] (q < 4) or v.b[q - 4]; its cosine and sine are element q of cs.a and cs.b
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float2 w = q < 4 ? v.a[q & 3] : v.b[q & 3];
              const float c = q & 1 ? cs.a[q >> 1].y : cs.a[q >> 1].x, s = q & 1 ? cs.b[q >> 1].y : cs.b[q >> 1].x;
              const float2 turned = make_float2(fmaf(w.x, c, -(w.y * s)), fmaf(w.y, c, w.x * s));
              if (q < 4) o.a[q & 3] = turned;
              else o.b[q & 3] = turned;
            }
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 minus = make_float2(-cs.b[j].x, -cs.b[j].y);
              o.a[j] = __ffma2_rn(v.a[j], cs.a[j], __fmul2_rn(v.b[j], minus));
              o.b[j] = __ffma2_rn(v.b[j], cs.a[j], __fmul2_rn(v.a[j], cs.b[j]));
            }
          }
          const int h = h0 + slot + k * step;
          if (MODE == NORM_TURN_GRAD) {
            if (!(active && h < h_end)) rstd[k] = 0.f;  // adds nothing to the gains' gradients
            Sixteen xh;
            open16(px[k], xh);
            const float2 r = twice(rstd[k]);
            float2 dot = make_float2(0.f, 0.f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              xh.a[j] = __fmul2_rn(xh.a[j], r);
              xh.b[j] = __fmul2_rn(xh.b[j], r);
              dg[kind][j] = __ffma2_rn(o.a[j], xh.a[j], dg[kind][j]);
              dg[kind][4 + j] = __ffma2_rn(o.b[j], xh.b[j], dg[kind][4 + j]);
              o.a[j] = __fmul2_rn(o.a[j], gain.a[j]);
              o.b[j] = __fmul2_rn(o.b[j], gain.b[j]);
              dot = __ffma2_rn(o.a[j], xh.a[j], dot);
              dot = __ffma2_rn(o.b[j], xh.b[j], dot);
            }
            float mean[1] = {dot.x + dot.y};
            head_sums(mean, sums);
            const float2 f = twice(-mean[0] * p.inv_d);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              o.a[j] = __fmul2_rn(r, __ffma2_rn(f, xh.a[j], o.a[j]));
              o.b[j] = __fmul2_rn(r, __ffma2_rn(f, xh.b[j], o.b[j]));
            }
          }
          if (active && h < h_end) store16(y + h * p.d, second, o);
        }
      }
    }
    if (RING) {
      __syncwarp();                                     // the row has been read
      if (lane == 0 && u + p.stages * next_unit < units) fetch_row(u + p.stages * next_unit, stage);
      if (++stage == p.stages) {
        stage = 0;
        parity ^= 1;
      }
    }
  }

  if (MODE == NORM_TURN_GRAD) {
    // this block's share of the gains' gradients: its heads are added in a fixed order
    const int groups = WARPS * p.side;
    if (RING) __syncthreads();                          // the rings are done with
    if (active) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float* to = share + ((warp * p.side + slot) * 2 + k) * p.d + c0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          *reinterpret_cast<float2*>(to + 2 * j) = dg[k][j];
          *reinterpret_cast<float2*>(to + second + 2 * j) = dg[k][4 + j];
        }
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.d; i += THREADS) {
      float sum = 0.f;
      for (int g = 0; g < groups; ++g) sum += share[g * 2 * p.d + i];
      p.partial[(int64_t)blockIdx.x * 2 * p.d + i] = sum;
    }
  }
}

// dq_gain[c], dk_gain[c] = sum of the blocks' shares, in a fixed order: 8 channels (a sector) to a block, 128 threads to
// a channel, all loads of a thread in flight together
constexpr int GAIN_THREADS = 1024, GAIN_CHANNELS = 8;
__global__ void __launch_bounds__(GAIN_THREADS)
gain_grad_kernel(const float* __restrict__ partial, int blocks, int d, float* __restrict__ dq_gain, float* __restrict__ dk_gain) {
  __shared__ float sums[GAIN_THREADS / 32][GAIN_CHANNELS];
  const int channel = threadIdx.x & (GAIN_CHANNELS - 1), part = threadIdx.x / GAIN_CHANNELS, i = blockIdx.x * GAIN_CHANNELS + channel;
  asm volatile("griddepcontrol.wait;" ::: "memory");     // the shares are written by the kernel before this one
  float sum = 0.f;
#pragma unroll 8
  for (int b = part; b < blocks; b += GAIN_THREADS / GAIN_CHANNELS) sum += partial[(int64_t)b * 2 * d + i];
  sum += __shfl_xor_sync(0xffffffffu, sum, 8);
  sum += __shfl_xor_sync(0xffffffffu, sum, 16);
  if ((threadIdx.x & 31) < GAIN_CHANNELS) sums[threadIdx.x >> 5][channel] = sum;
  __syncthreads();
  if (threadIdx.x < GAIN_CHANNELS) {
    sum = 0.f;
#pragma unroll
    for (int b = 0; b < GAIN_THREADS / 32; ++b) sum += sums[b][channel];
    (i < d ? dq_gain : dk_gain)[i < d ? i : i - d] = sum;
  }
}

struct Shape { int split, grid, stages; size_t smem; };

Shape shape_of(int mode, int rows, int heads, int d, bool full, size_t es, int sms) {
  Shape s;
  s.stages = 0;
  const int side = 32 / (d / (full ? 16 : CH));
  // a row's heads are shared by more warps where the rows alone would not fill the device
  s.split = 1;
  while (s.split < 8 && (int64_t)rows * s.split < (int64_t)sms * 16 && heads > 2 * s.split * side) s.split *= 2;
  const int64_t blocks = ((int64_t)rows * s.split + WARPS - 1) / WARPS, most = (int64_t)sms * (mode == NORM_TURN_GRAD ? 4 : 32);
  s.grid = (int)(blocks < most ? blocks : most);
  s.smem = mode == NORM_TURN_GRAD ? (size_t)WARPS * side * 2 * d * sizeof(float) : 0;
  // a ring of two rows or more for every warp, if it leaves room for three (gradients) or four blocks on an SM and
  // every warp has a few rows to fetch ahead
  const size_t stage = (size_t)WARPS * heads * d * es * (mode == NORM_TURN_GRAD ? 2 : 1), room = (mode == NORM_TURN_GRAD ? 72 : 54) * 1024;
  // (rotation alone is faster without it: 73 against 86 us at 36864 rows of 24 heads of 128)
  if (mode != TURN && full && s.split == 1 && 2 * stage <= room && (int64_t)rows >= (int64_t)sms * 32) {
    s.stages = (int)(room / stage < 4 ? room / stage : 4);
    if (s.smem < s.stages * stage) s.smem = s.stages * stage;
    const int64_t resident = (int64_t)sms * (mode == NORM_TURN_GRAD ? 3 : 4);
    s.grid = (int)(blocks < resident ? blocks : resident);
  }
  return s;
}

template <typename T, bool IL, int MODE>
cudaError_t launch_ring(const RopeNormArgs& a, const Shape& s, cudaStream_t stream) {
  constexpr int STEPS = MODE == NORM_TURN_GRAD ? 1 : sizeof(T) == 4 ? 2 : 3;
  static PerDeviceFlag done;
  if (cudaError_t e = ensure_dynamic_smem(done, rope_norm_full_kernel<T, IL, MODE, STEPS, true>, 100 * 1024)) return e;
  rope_norm_full_kernel<T, IL, MODE, STEPS, true><<<s.grid, THREADS, s.smem, stream>>>(a);
  return cudaGetLastError();
}
template <typename T, int MODE>
cudaError_t launch_mode(const RopeNormArgs& a, bool interleaved, const Shape& s, cudaStream_t stream) {
  constexpr int HEADS = sizeof(T) == 4 || MODE == NORM_TURN_GRAD ? 2 : 4;
  constexpr int STEPS = sizeof(T) == 4 ? (MODE == NORM_TURN_GRAD ? 1 : 2) : MODE == NORM_TURN_GRAD ? 2 : 3;
  if (2 * a.n_pairs == a.d) {
    if constexpr (MODE != TURN)
      if (a.stages > 0) return interleaved ? launch_ring<T, true, MODE>(a, s, stream) : launch_ring<T, false, MODE>(a, s, stream);
    if (interleaved) rope_norm_full_kernel<T, true, MODE, STEPS, false><<<s.grid, THREADS, s.smem, stream>>>(a);
    else rope_norm_full_kernel<T, false, MODE, STEPS, false><<<s.grid, THREADS, s.smem, stream>>>(a);
  } else if (interleaved || a.n_pairs == 0) rope_norm_kernel<T, INTERLEAVED, MODE, HEADS><<<s.grid, THREADS, s.smem, stream>>>(a);
  else if (a.n_pairs % CH == 0) rope_norm_kernel<T, HALVES_BY_LANES, MODE, HEADS><<<s.grid, THREADS, s.smem, stream>>>(a);
  else rope_norm_kernel<T, HALVES_ANY, MODE, HEADS><<<s.grid, THREADS, s.smem, stream>>>(a);
  return cudaGetLastError();
}

}  // namespace

size_t qk_norm_rope_backward_bytes(int d) {
  return (size_t)4 * MAX_SMS * 2 * d * sizeof(float);      // one share for each block of the largest grid
}

cudaError_t launch_rope_norm(const RopeNormCall& c, cudaStream_t s) {
  if (c.rows <= 0 || c.heads <= 0) return cudaSuccess;
  const int sms = current_device_sm_count();
  if (sms < 1 || sms > MAX_SMS) return cudaErrorInvalidDevice;
  const int mode = c.dy ? NORM_TURN_GRAD : c.q_gain ? NORM_TURN : TURN;
  RopeNormArgs a{};
  a.rows = c.rows; a.heads = c.heads; a.q_heads = c.q_heads; a.d = c.d;
  a.inv_d = 1.0f / (float)c.d;
  if (c.rope) {
    for (int i = 0; i < c.rope->axes; ++i) a.first_pair[i + 1] = a.first_pair[i] + c.rope->pairs[i];
    a.n_pairs = a.first_pair[c.rope->axes];
    a.positions = c.rope->positions; a.freqs = c.rope->freqs;
  }
  a.turn_sign = c.inverse != (mode == NORM_TURN_GRAD) ? -1.f : 1.f;
  a.eps = c.eps; a.q_gain = c.q_gain; a.k_gain = c.k_gain;
  a.x = c.x; a.ldx = c.ldx; a.dy = c.dy; a.lddy = c.lddy; a.y = c.y; a.ldy = c.ldy; a.partial = c.partial;
  const bool full = 2 * a.n_pairs == c.d;
  a.lanes = c.d / (full ? 16 : CH); a.side = 32 / a.lanes;
  const Shape sh = shape_of(mode, c.rows, c.heads, c.d, full, c.act_bf16 ? 2 : 4, sms);
  a.split = sh.split; a.stages = sh.stages; a.dev_status = c.dev_status;
  const bool il = c.rope && c.rope->interleaved;
  if (c.act_bf16)
    return mode == TURN ? launch_mode<bf16, TURN>(a, il, sh, s) : mode == NORM_TURN ? launch_mode<bf16, NORM_TURN>(a, il, sh, s)
                                                                                   : launch_mode<bf16, NORM_TURN_GRAD>(a, il, sh, s);
  return mode == TURN ? launch_mode<float, TURN>(a, il, sh, s) : mode == NORM_TURN ? launch_mode<float, NORM_TURN>(a, il, sh, s)
                                                                                  : launch_mode<float, NORM_TURN_GRAD>(a, il, sh, s);
}

cudaError_t launch_gain_grad(const RopeNormCall& c, float* dq_gain, float* dk_gain, cudaStream_t s) {
  const int sms = current_device_sm_count();
  if (sms < 1 || sms > MAX_SMS) return cudaErrorInvalidDevice;
  int n_pairs = 0;
  for (int i = 0; c.rope && i < c.rope->axes; ++i) n_pairs += c.rope->pairs[i];
  const bool full = 2 * n_pairs == c.d;
  const int blocks = c.rows > 0 ? shape_of(NORM_TURN_GRAD, c.rows, c.heads, c.d, full, c.act_bf16 ? 2 : 4, sms).grid : 0;   // no rows: the gradients are zero
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(2 * c.d / GAIN_CHANNELS);                   // (d is a multiple of 16)
  cfg.blockDim = dim3(GAIN_THREADS);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];                           // its launch overlaps the end of the kernel before it
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, gain_grad_kernel, (const float*)c.partial, blocks, c.d, dq_gain, dk_gain);
}

}  // namespace vit
