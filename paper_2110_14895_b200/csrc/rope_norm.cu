// Rotary positions on several axes, alone or behind the root-mean-square norm of every query and
// key head, and the gradients of the latter.
//
//   y = R x                                  pair i of a head turned by positions[axis(i)][row] * freqs[i]
//   y = R (g x / sqrt(mean(x^2) + eps))      norm, gain, rotation
//   u = R^T dy, xh = x rstd, w = g u:        dx = rstd (w - xh mean(w xh)),  dg = sum over rows and heads of u xh
//
// All of them are bound by HBM: every element is read once and written once, in 16-byte pieces.  A head
// belongs to a power of two of neighbouring lanes, eight channels to a lane, so that the sums of the norm
// are a few shuffles and nothing of a head leaves its warp.  The angles of a row are shared by its heads:
// a block turns them into cosines and sines once, in shared memory, and every lane keeps those of its
// eight channels in registers while it walks over the row's heads.
#include "vit_internal.h"

#include <cmath>

namespace vit {

namespace {

constexpr int THREADS = 256;
constexpr int CH = 8;                       // channels of a lane
constexpr int MAX_SMS = 256;

enum Rotation { INTERLEAVED = 0, HALVES_BY_LANES = 1, HALVES_ANY = 2 };
enum Mode { TURN = 0, NORM_TURN = 1, NORM_TURN_GRAD = 2 };

struct RopeNormArgs {
  int rows, heads, q_heads, d;
  int n_pairs, axes, first_pair[5];         // axis a turns the pairs [first_pair[a], first_pair[a + 1])
  int rows_per_block, row_blocks;
  float turn_sign;                          // +1: by the angle, -1: back
  float eps;
  const int32_t* positions;                 // [axes][rows]
  const float* freqs;                       // [n_pairs]
  const float *q_gain, *k_gain;             // [d]
  const void* x;  int64_t ldx;
  const void* dy; int64_t lddy;             // NORM_TURN_GRAD
  void* y;        int64_t ldy;              // y, or dx
  float* partial;                           // NORM_TURN_GRAD: [gridDim.x][2][d]
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
__device__ __forceinline__ float to_f(bf16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(float v) { return v; }

// Cosine and sine of position * freq.  The product of a 31-bit position and a 24-bit frequency is exact
// in 64 bits; whole turns are taken off there, so that far positions keep their angle to 32 bits.
__device__ __forceinline__ float2 turn_of(int32_t position, float freq) {
  const double turns = (double)position * (double)freq * 0.15915494309189533577;
  float s, c;
  sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
  return make_float2(c, s);
}

// One warp-aligned group of G lanes per (row, head).  HEADS heads of a group are in flight at a time.
template <typename T, int G, int ROT, int MODE, int HEADS>
__global__ void __launch_bounds__(THREADS)
rope_norm_kernel(const RopeNormArgs p) {
  extern __shared__ float2 table[];                     // [rows_per_block][n_pairs]
  constexpr int GROUPS = THREADS / G;
  const int lane = threadIdx.x % G, group = threadIdx.x / G;
  const int per_row = GROUPS / p.rows_per_block;        // groups that share a row's heads
  const int row_in_block = group / per_row, first_head = group % per_row;
  const int c0 = lane * CH;
  const bool active = c0 < p.d;
  const int n = p.n_pairs;
  const unsigned full = 0xffffffffu;

  float qg[CH], kg[CH], dqg[CH], dkg[CH];
#pragma unroll
  for (int j = 0; j < CH; ++j) {
    qg[j] = MODE != TURN && active ? p.q_gain[c0 + j] : 0.f;
    kg[j] = MODE != TURN && active ? p.k_gain[c0 + j] : 0.f;
    dqg[j] = dkg[j] = 0.f;
  }

  for (int rb = blockIdx.x; rb < p.row_blocks; rb += gridDim.x) {
    const int64_t row0 = (int64_t)rb * p.rows_per_block;
    if (rb != (int)blockIdx.x) __syncthreads();         // the table of the last rows is no longer read
    for (int i = threadIdx.x; i < p.rows_per_block * n; i += THREADS) {
      const int r = i / n, pair = i - r * n;
      if (row0 + r < p.rows) {
        int axis = 0;
        while (pair >= p.first_pair[axis + 1]) ++axis;
        table[i] = turn_of(p.positions[(int64_t)axis * p.rows + row0 + r], p.freqs[pair]);
      }
    }
    __syncthreads();
    const int64_t row = row0 + row_in_block;
    const bool row_ok = row < p.rows;
    // out[j] = v[j] * cs[j] + partner(v)[j] * sn[j] where the channel turns
    float cs[CH], sn[CH];
    int partner[CH];                                    // HALVES_ANY: the partner's channel
    uint32_t turning = 0;                               // bit j: channel j turns
#pragma unroll
    for (int j = 0; j < CH; ++j) {
      const int c = c0 + j;
      int pair;
      float sign;
      if (ROT == INTERLEAVED) { pair = c >> 1; sign = (c & 1) ? 1.f : -1.f; partner[j] = c ^ 1; }
      else if (c < n) { pair = c; sign = -1.f; partner[j] = c + n; }
      else { pair = c - n; sign = 1.f; partner[j] = c - n; }
      const bool turns = active && row_ok && pair < n;
      const float2 t = turns ? table[row_in_block * n + pair] : make_float2(1.f, 0.f);
      cs[j] = t.x;
      sn[j] = sign * p.turn_sign * t.y;
      if (turns) turning |= 1u << j; else partner[j] = c;
    }
    // HALVES_BY_LANES: the partner's eight channels are those of one other lane of the group
    const int partner_lane = active ? partner[0] / CH : lane;

    for (int hb = 0; hb < p.heads; hb += per_row * HEADS) {   // as many turns for every group: its warp shuffles
      const int h0 = hb + first_head;
      Piece<T> px[HEADS], pd[HEADS];
      bool on[HEADS];
#pragma unroll
      for (int k = 0; k < HEADS; ++k) {                 // all loads in flight before the first use
        const int h = h0 + k * per_row;
        on[k] = active && row_ok && h < p.heads;
        if (on[k]) {
          load_piece(px[k], static_cast<const T*>(p.x) + row * p.ldx + (int64_t)h * p.d + c0);
          if (MODE == NORM_TURN_GRAD) load_piece(pd[k], static_cast<const T*>(p.dy) + row * p.lddy + (int64_t)h * p.d + c0);
        }
      }
#pragma unroll
      for (int k = 0; k < HEADS; ++k) {
        const int h = h0 + k * per_row;
        const bool is_q = h < p.q_heads;
        float x[CH] = {}, o[CH];
        if (on[k]) unpack(px[k], x);
        float rstd = 1.f;
        if (MODE != TURN) {
          float sq = 0.f;
#pragma unroll
          for (int j = 0; j < CH; ++j) sq = fmaf(x[j], x[j], sq);
#pragma unroll
          for (int s = G / 2; s > 0; s >>= 1) sq += __shfl_xor_sync(full, sq, s, G);
          rstd = 1.0f / sqrtf(sq / (float)p.d + p.eps);
        }
        float v[CH] = {};                               // what is turned
        if (MODE == NORM_TURN_GRAD) {
          if (on[k]) unpack(pd[k], v);
        } else {
#pragma unroll
          for (int j = 0; j < CH; ++j) v[j] = MODE == NORM_TURN ? x[j] * rstd * (is_q ? qg[j] : kg[j]) : x[j];
        }
#pragma unroll
        for (int j = 0; j < CH; ++j) {
          float other;
          if (ROT == INTERLEAVED) {
            other = v[j ^ 1];
          } else if (ROT == HALVES_BY_LANES) {
            other = __shfl_sync(full, v[j], partner_lane, G);
          } else {
            // the partner lies at any offset: read it again (it is in L1), before this head is written
            other = 0.f;
            if (on[k]) {
              const int c = partner[j];
              if (MODE == NORM_TURN_GRAD) {
                other = to_f(static_cast<const T*>(p.dy)[row * p.lddy + (int64_t)h * p.d + c]);
              } else {
                other = to_f(static_cast<const T*>(p.x)[row * p.ldx + (int64_t)h * p.d + c]);
                if (MODE == NORM_TURN) other *= rstd * (is_q ? p.q_gain[c] : p.k_gain[c]);
              }
            }
          }
          // a channel that does not turn is passed on as it is, whatever its partner holds
          o[j] = turning >> j & 1 ? fmaf(v[j], cs[j], other * sn[j]) : v[j];
        }
        if (MODE == NORM_TURN_GRAD) {
          float dot = 0.f;
#pragma unroll
          for (int j = 0; j < CH; ++j) {
            const float xh = x[j] * rstd;
            const float dg = o[j] * xh;
            if (is_q) dqg[j] += dg; else dkg[j] += dg;   // lanes without a head hold x = 0
            o[j] *= is_q ? qg[j] : kg[j];
            dot = fmaf(o[j], xh, dot);
          }
#pragma unroll
          for (int s = G / 2; s > 0; s >>= 1) dot += __shfl_xor_sync(full, dot, s, G);
          const float mean = dot / (float)p.d;
#pragma unroll
          for (int j = 0; j < CH; ++j) o[j] = rstd * (o[j] - x[j] * rstd * mean);
        }
        if (ROT == HALVES_ANY) __syncwarp();             // in place: every lane has read before any writes
        if (on[k]) store_piece(static_cast<T*>(p.y) + row * p.ldy + (int64_t)h * p.d + c0, o);
      }
    }
  }

  if (MODE == NORM_TURN_GRAD) {
    // this block's share of the gains' gradients: its groups are added in a fixed order
    __syncthreads();
    float* share = reinterpret_cast<float*>(table);      // [GROUPS][2][d]
    if (active) {
#pragma unroll
      for (int j = 0; j < CH; ++j) {
        share[(group * 2 + 0) * p.d + c0 + j] = dqg[j];
        share[(group * 2 + 1) * p.d + c0 + j] = dkg[j];
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * p.d; i += THREADS) {
      float sum = 0.f;
      for (int g = 0; g < GROUPS; ++g) sum += share[g * 2 * p.d + i];
      p.partial[(int64_t)blockIdx.x * 2 * p.d + i] = sum;
    }
  }
}

// dq_gain[c], dk_gain[c] = sum of the blocks' shares, in a fixed order: one warp per channel
__global__ void __launch_bounds__(THREADS)
gain_grad_kernel(const float* __restrict__ partial, int blocks, int d, float* __restrict__ dq_gain, float* __restrict__ dk_gain) {
  const int i = (int)((blockIdx.x * THREADS + threadIdx.x) >> 5), lane = threadIdx.x & 31;
  if (i >= 2 * d) return;
  float sum = 0.f;
  for (int b = lane; b < blocks; b += 32) sum += partial[(int64_t)b * 2 * d + i];
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
  if (lane == 0) (i < d ? dq_gain : dk_gain)[i < d ? i : i - d] = sum;
}

struct Shape { int rows_per_block, row_blocks, grid; size_t smem; };

Shape shape_of(int mode, int rows, int heads, int d, int n_pairs, int G, int sms) {
  Shape s;
  const int groups = THREADS / G;
  // As many rows to a block as leave each group about eight heads of a row, so that a row's angles
  // serve many heads; fewer rows where the call would not fill the device otherwise.
  int r = 1;
  while (r * 2 <= groups && heads * r * 2 <= groups * 8 && (int64_t)rows / (r * 2) >= 2 * sms) r *= 2;
  s.rows_per_block = r;
  s.row_blocks = (rows + r - 1) / r;
  s.grid = s.row_blocks;
  if (mode == NORM_TURN_GRAD && s.grid > 4 * sms) s.grid = 4 * sms;   // one share of the gains' gradients per block
  s.smem = (size_t)r * n_pairs * sizeof(float2);
  if (mode == NORM_TURN_GRAD && s.smem < (size_t)groups * 2 * d * 4) s.smem = (size_t)groups * 2 * d * 4;
  return s;
}

template <typename T, int G, int ROT, int MODE>
cudaError_t launch_variant(RopeNormArgs& a, const Shape& s, cudaStream_t stream) {
  constexpr int HEADS = MODE == NORM_TURN_GRAD ? 2 : 4;
  rope_norm_kernel<T, G, ROT, MODE, HEADS><<<s.grid, THREADS, s.smem, stream>>>(a);
  return cudaGetLastError();
}
template <typename T, int G, int MODE>
cudaError_t launch_rot(RopeNormArgs& a, bool interleaved, const Shape& s, cudaStream_t stream) {
  if (interleaved || a.n_pairs == 0) return launch_variant<T, G, INTERLEAVED, MODE>(a, s, stream);
  if (a.n_pairs % CH == 0) return launch_variant<T, G, HALVES_BY_LANES, MODE>(a, s, stream);
  return launch_variant<T, G, HALVES_ANY, MODE>(a, s, stream);
}
template <typename T, int MODE>
cudaError_t launch_lanes(RopeNormArgs& a, bool interleaved, const Shape& s, int G, cudaStream_t stream) {
  switch (G) {
    case 2: return launch_rot<T, 2, MODE>(a, interleaved, s, stream);
    case 4: return launch_rot<T, 4, MODE>(a, interleaved, s, stream);
    case 8: return launch_rot<T, 8, MODE>(a, interleaved, s, stream);
    default: return launch_rot<T, 16, MODE>(a, interleaved, s, stream);
  }
}

int lanes_of(int d) {
  int g = 2;
  while (g * CH < d) g *= 2;
  return g;
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
  if (c.rope) {
    a.axes = c.rope->axes;
    for (int i = 0; i < a.axes; ++i) a.first_pair[i + 1] = a.first_pair[i] + c.rope->pairs[i];
    a.n_pairs = a.first_pair[a.axes];
    a.positions = c.rope->positions; a.freqs = c.rope->freqs;
  }
  a.turn_sign = c.inverse != (mode == NORM_TURN_GRAD) ? -1.f : 1.f;
  a.eps = c.eps; a.q_gain = c.q_gain; a.k_gain = c.k_gain;
  a.x = c.x; a.ldx = c.ldx; a.dy = c.dy; a.lddy = c.lddy; a.y = c.y; a.ldy = c.ldy; a.partial = c.partial;
  const int G = lanes_of(c.d);
  const Shape sh = shape_of(mode, c.rows, c.heads, c.d, a.n_pairs, G, sms);
  a.rows_per_block = sh.rows_per_block; a.row_blocks = sh.row_blocks;
  const bool il = c.rope && c.rope->interleaved;
  cudaError_t e;
  if (c.act_bf16)
    e = mode == TURN ? launch_lanes<bf16, TURN>(a, il, sh, G, s) : mode == NORM_TURN ? launch_lanes<bf16, NORM_TURN>(a, il, sh, G, s)
                                                                                     : launch_lanes<bf16, NORM_TURN_GRAD>(a, il, sh, G, s);
  else
    e = mode == TURN ? launch_lanes<float, TURN>(a, il, sh, G, s) : mode == NORM_TURN ? launch_lanes<float, NORM_TURN>(a, il, sh, G, s)
                                                                                      : launch_lanes<float, NORM_TURN_GRAD>(a, il, sh, G, s);
  return e;
}

cudaError_t launch_gain_grad(const RopeNormCall& c, float* dq_gain, float* dk_gain, cudaStream_t s) {
  const int sms = current_device_sm_count();
  if (sms < 1 || sms > MAX_SMS) return cudaErrorInvalidDevice;
  int blocks = 0;                                        // no rows: the gradients are zero
  if (c.rows > 0) blocks = shape_of(NORM_TURN_GRAD, c.rows, c.heads, c.d, 0, lanes_of(c.d), sms).grid;
  gain_grad_kernel<<<(2 * c.d * 32 + THREADS - 1) / THREADS, THREADS, 0, s>>>(c.partial, blocks, c.d, dq_gain, dk_gain);
  return cudaGetLastError();
}

}  // namespace vit
