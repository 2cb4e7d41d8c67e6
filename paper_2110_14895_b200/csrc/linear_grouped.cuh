// What the kernels of linear layers by group share: where a group's rows lie, how the work is cut, GELU and its slope.
#pragma once
#include "vit_internal.h"
#include "sm100_ptx.cuh"

namespace vit {

// The offsets live on the device and are the caller's: a group whose rows are not in order or not inside the buffer is
// skipped, and the status word says so.  Without offsets there is one group, of all rows.
__device__ __forceinline__ bool group_rows(const GroupedShape& p, int g, int& begin, int& end) {
  begin = 0;
  end = p.rows;
  if (p.offsets) {
    begin = p.offsets[g];
    end = p.offsets[g + 1];
  }
  return begin >= 0 && end >= begin && end <= p.rows;
}

__device__ __forceinline__ int warp_scan(int v, int lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int lower = __shfl_up_sync(0xffffffffu, v, d);
    if (lane >= d) v += lower;
  }
  return v;
}

// Which group a unit of work belongs to.  Units are numbered group after group; a warp looks at 32 groups at a time and
// asks for ever larger numbers.  All lanes call together and get the same answer.  Units fit 32 bits (checked on the host).
struct GroupAt { int group, begin, end, before; };               // its rows, and the units before it
template <typename Count>                                        // Count: (rows of a group) -> its units
struct GroupWalk {
  const GroupedShape& p;
  Count count;
  int lane, g0, begin, end;
  int base, upto, chunk;                                          // units before the 32 groups, up to this lane's group, of all 32

  __device__ __forceinline__ GroupWalk(const GroupedShape& shape, Count c, int lane_) : p(shape), count(c), lane(lane_), g0(0), base(0) { load(); }
  __device__ __forceinline__ void restart() {
    g0 = 0;
    base = 0;
    load();
  }
  __device__ __forceinline__ void load() {
    const int g = g0 + lane;
    int n = 0;
    begin = end = 0;
    if (g < p.groups) {
      if (group_rows(p, g, begin, end)) n = count(end - begin);
      else begin = end = 0;
    }
    upto = warp_scan(n, lane);
    chunk = __shfl_sync(0xffffffffu, upto, 31);
  }
  __device__ __forceinline__ bool find(int unit, GroupAt& at) {
    while (unit - base >= chunk) {
      if (g0 + 32 >= p.groups) return false;
      base += chunk;
      g0 += 32;
      load();
    }
    const uint32_t later = __ballot_sync(0xffffffffu, base + upto > unit);
    const int who = __ffs((int)later) - 1;
    at.group = g0 + who;
    at.begin = __shfl_sync(0xffffffffu, begin, who);
    at.end = __shfl_sync(0xffffffffu, end, who);
    const int before = __shfl_up_sync(0xffffffffu, upto, 1);
    at.before = base + (who == 0 ? 0 : __shfl_sync(0xffffffffu, before, who));
    return true;
  }
};
__device__ __forceinline__ int warp_total(int v) { return __reduce_add_sync(0xffffffffu, v); }
__device__ __forceinline__ void report_bad_groups(const GroupedShape& p, int* dev_status, int lane) {
  for (int g = lane; g < p.groups; g += 32) {
    int begin, end;
    if (!group_rows(p, g, begin, end)) atomicExch(dev_status, (int)VIT_ERR_OFFSETS);
  }
}

// Tiles of `span` rows by `across` columns' tiles.
struct TileCount {
  int span, across;
  __device__ __forceinline__ int operator()(int rows) const { return (rows + span - 1) / span * across; }
};

// The weights' gradients sum over a group's rows, tile by tile of [out][in], 64 rows to a unit (a group without rows has one
// for every tile: its zeros).  Tiles are numbered group after group.  Whole rounds of them go to the blocks in turn, tile i to
// block i mod blocks, so that the blocks are in the same group at the same rows at a time and find them in L2 (in stretches
// of neighbouring tiles all groups were read at once: 1.1 GB from memory for 0.26, and 213 us, at 25216 rows of 16 groups).
// The other tiles' units, with several groups a round's at least, lie in one line, of which a block gets as much as makes its
// work the mean: groups of any lengths come out even, and a long sum with few tiles is cut between all blocks.  A block's first
// and last tile there may be parts; each part has one owner, and the parts are joined in the order of their rows.
// Parts begin in the middle where that brings all blocks to the same rows modulo a share: at a time t of its share a block is
// at unit t + k share of its tile, for some k.
// Blocks at most; units of a share of the line at least, unless there are fewer tiles than blocks (grouped_dw_plan may ask for
// more): a unit takes 0.3 us on the tensor cores, 5 us on the fp32 pipes, and a part of a tile 2 us and more.
constexpr int DW_BLOCKS = 148, DW_BLOCKS_F32 = 296, DW_ROWS = 64, DW_LEAST = 8, DW_LEAST_F32 = 1;
struct SumCount {
  int tiles;
  bool whole;                                                    // counts tiles, not units
  static __device__ __forceinline__ int of(int rows) { return rows > DW_ROWS ? (rows + DW_ROWS - 1) / DW_ROWS : 1; }
  __device__ __forceinline__ int operator()(int rows) const { return tiles * (whole ? 1 : of(rows)); }
};
// What a block does: tiles self, self + blocks, ... below `round`, then units [begin, end) of all.
struct Share { int round, begin, end, beat; };                  // beat: the mean share
// begins: of all blocks in the line (units of all), and behind the last one its end; what a second kernel needs.
constexpr int DW_TABLE = DW_BLOCKS_F32 + 1, DW_SCRATCH = 2 * DW_TABLE;        // numbers; of shared memory while the shares are found

// All threads of a block, which get the same answer in every block.  cuts: whether tiles may be cut.
__device__ __forceinline__ Share find_share(const GroupedShape& p, int tiles, int blocks, int self, int least, int cuts, int* scratch, int* table) {
  const int lane = threadIdx.x & 31;
  int total = 0, whole = 0;
  for (int g = lane; g < p.groups; g += 32) {
    int begin, end;
    if (group_rows(p, g, begin, end)) {
      total += SumCount::of(end - begin);
      ++whole;
    }
  }
  total = warp_total(total) * tiles;
  whole = warp_total(whole) * tiles;
  if (cuts == 0) return Share{whole, 0, 0, 1};                   // all tiles go round
  const int rounds = whole / blocks, round = (p.groups == 1 ? rounds : rounds > 0 ? rounds - 1 : 0) * blocks;
  if (round == 0) {
    // the same to each, but to no more blocks than get something to do
    const int wanted = max(total / least, whole), used = min(max(wanted, 1), blocks);
    const double each = (double)total / used;
    auto begin = [&](int c) { return c >= used ? total : (int)(each * c); };
    if (table && self == 0)
      for (int c = threadIdx.x; c <= blocks; c += (int)blockDim.x) table[c] = begin(c);
    return Share{0, begin(self), begin(self + 1), max((int)each, 1)};
  }
  int *loads = scratch, *begins = scratch + DW_TABLE;
  for (int c = threadIdx.x; c < blocks; c += (int)blockDim.x) loads[c] = 0;
  __syncthreads();
  {
    // units that go round to block c: of a group's tiles [t0, t1) those that are c modulo the blocks
    const int slices = max((int)blockDim.x / blocks, 1), slice = (int)threadIdx.x / blocks;
    for (int c = (int)threadIdx.x % blocks; c < blocks && slice < slices; c += slices > 1 ? blocks : (int)blockDim.x) {
      const int per = (p.groups + slices - 1) / slices;
      // every group has `tiles` of them: q or q + 1 are c modulo the blocks, by where its first one lies
      const int q = tiles / blocks, r = tiles % blocks;
      int sum = 0, at = 0;                                       // at: t0 modulo the blocks
      for (int g = 0, t0 = 0; g < min(p.groups, (slice + 1) * per) && t0 < round; ++g) {
        int begin, end;
        if (!group_rows(p, g, begin, end)) continue;
        if (g >= slice * per) {
          const int from = c >= at ? c - at : c - at + blocks;   // of the first of them behind t0
          const int n = t0 + tiles <= round ? q + (from < r ? 1 : 0) : (round - t0 - from + blocks - 1) / blocks;
          sum += n * SumCount::of(end - begin);
        }
        t0 += tiles;
        at += r;
        if (at >= blocks) at -= blocks;
      }
      atomicAdd(&loads[c], sum);                                 // whole numbers: any order
    }
    __syncthreads();
  }
  if (threadIdx.x < 32) {
    constexpr int N = (DW_BLOCKS_F32 + 31) / 32;
    int load[N], done = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int c = lane + 32 * i;
      load[i] = c < blocks ? loads[c] : INT32_MAX;
      if (c < blocks) done += load[i];
    }
    done = warp_total(done);
    const int line = total - done, left = whole - round, wanted = max(line / least, left);
    // a short line goes to as many blocks as get something to do, the same to each; else the line fills the blocks up to a
    // level, and those above it get nothing
    const bool few = wanted < blocks;
    const int used = few ? max(wanted, 1) : blocks;
    int level = (int)(((int64_t)total + blocks - 1) / blocks), shares = used;
    for (int k = 0; !few && k < 16; ++k) {
      int sum = 0, open = 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (load[i] < level) {
          sum += level - load[i];
          ++open;
        }
      shares = warp_total(sum);
      open = warp_total(open);
      if (shares <= line + open || k == 15) break;
      level -= (shares - line) / open;
    }
    const double each = shares > 0 ? (double)line / shares : 0.0;
    int before = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (32 * i >= blocks) break;
      const int c = lane + 32 * i, mine = few ? (c < used ? 1 : 0) : load[i] < level ? level - load[i] : 0;
      const int upto = warp_scan(mine, lane);
      if (c < blocks) begins[c] = done + (int)(each * (before + upto - mine));
      before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0) {
      begins[blocks] = total;
      loads[0] = max(line / used, 1);
    }
  }
  __syncthreads();
  const Share share{round, begins[self], begins[self + 1], loads[0]};
  if (table && self == 0)
    for (int c = threadIdx.x; c <= blocks; c += (int)blockDim.x) table[c] = begins[c];
  return share;                                                  // (the scratch is in use until the block has met again)
}

// A block's work on one tile: units [from, to) of `all`.  slot: where a part's sums are kept, the share's first or last.
struct Part {
  int group, begin, end, tile, from, to, all, first;             // first: the unit that it begins with
  __device__ __forceinline__ int unit(int i) const { return first + i < to ? first + i : first + i - (to - from); }
  __device__ __forceinline__ bool whole() const { return from == 0 && to == all; }
  __device__ __forceinline__ int slot() const { return from == 0 ? 1 : 0; }
  __device__ __forceinline__ int blocks() const { return end > begin ? to - from : 0; }      // of 64 rows
};
// One part after the other; one warp, all lanes.
struct PartWalk {
  GroupWalk<SumCount> walk;
  Share share;
  int at, blocks;
  __device__ __forceinline__ PartWalk(const GroupedShape& p, int tiles, int lane, const Share& s, int self, int blocks_)
      : walk(p, SumCount{tiles, s.round > 0}, lane), share(s), at(s.round > 0 ? self : s.begin), blocks(blocks_) {}
  __device__ __forceinline__ bool next(Part& part) {
    GroupAt g;
    if (walk.count.whole) {
      if (at < share.round && walk.find(at, g)) {
        part = Part{g.group, g.begin, g.end, at - g.before, 0, 0, SumCount::of(g.end - g.begin), 0};
        part.to = part.all;
        at += blocks;
        return true;
      }
      walk.count.whole = false;
      walk.restart();
      at = share.begin;
    }
    if (at >= share.end || !walk.find(at, g)) return false;
    const int all = SumCount::of(g.end - g.begin);
    const int local = at - g.before, tile = local / all;
    part = Part{g.group, g.begin, g.end, tile, local - tile * all, 0, all, 0};
    part.to = min(all, part.from + share.end - at);
    // the first unit in it that is the time of the share, modulo the beat
    const int late = (part.from - (at - share.begin)) % share.beat;
    part.first = part.from + (late > 0 ? share.beat - late : -late);
    if (part.first >= part.to) part.first = part.from;
    at += part.to - part.from;
    return true;
  }
};

// gelu(v) = v Phi(v) and its slope Phi(v) + v phi(v), with a = |v| and
//   erfc(a / sqrt 2) = (a1 t + ... + a5 t^5) e,  t = 1 / (1 + p a / sqrt 2),  e = exp(-a^2 / 2)
// (Abramowitz & Stegun 7.1.26, |error| <= 1.5e-7), two values at a time.  a is held at 24, where e is zero in 32 bits, so
// that infinities give their limits.
struct Gelu2 { float2 half_erfc, e, a; };       // 0.5 erfc(a / sqrt 2), exp(-a^2 / 2), |v|
__device__ __forceinline__ Gelu2 gelu_parts(float2 v) {
  Gelu2 g;
  g.a = make_float2(fabsf(v.x), fabsf(v.y));
  g.a.x = g.a.x > 24.f ? 24.f : g.a.x;          // (a value that is not a number stays one)
  g.a.y = g.a.y > 24.f ? 24.f : g.a.y;
  const float kp = 0.3275911f * 0.70710678118654752440f;
  const float2 den = __ffma2_rn(make_float2(kp, kp), g.a, make_float2(1.0f, 1.0f));
  float2 t;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t.x) : "f"(den.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(t.y) : "f"(den.y));
  const float ke = -0.5f * 1.4426950408889634f;
  const float2 arg = __fmul2_rn(__fmul2_rn(g.a, g.a), make_float2(ke, ke));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(g.e.x) : "f"(arg.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(g.e.y) : "f"(arg.y));
  const float c5 = 0.5f * 1.061405429f, c4 = 0.5f * -1.453152027f, c3 = 0.5f * 1.421413741f, c2 = 0.5f * -0.284496736f,
              c1 = 0.5f * 0.254829592f;
  float2 q = __ffma2_rn(make_float2(c5, c5), t, make_float2(c4, c4));
  q = __ffma2_rn(q, t, make_float2(c3, c3));
  q = __ffma2_rn(q, t, make_float2(c2, c2));
  q = __ffma2_rn(q, t, make_float2(c1, c1));
  g.half_erfc = __fmul2_rn(__fmul2_rn(q, t), g.e);
  return g;
}
__device__ __forceinline__ float2 gelu_2(float2 v) {
  const Gelu2 g = gelu_parts(v);
  return __ffma2_rn(make_float2(-g.a.x, -g.a.y), g.half_erfc, make_float2(fmaxf(v.x, 0.f), fmaxf(v.y, 0.f)));
}
__device__ __forceinline__ float2 gelu_slope_2(float2 v) {
  const Gelu2 g = gelu_parts(v);
  const float k = -0.39894228040143267794f;     // -1 / sqrt(2 pi)
  const float2 below = __ffma2_rn(__fmul2_rn(make_float2(k, k), g.a), g.e, g.half_erfc);       // the slope at -a; 1 - it at a
  return make_float2(v.x > 0.f ? 1.f - below.x : below.x, v.y > 0.f ? 1.f - below.y : below.y);
}
// in 32 bits, with the library's error function
__device__ __forceinline__ float gelu_f32(float v) {
  return v < -24.f ? -0.f : v > 24.f ? v : 0.5f * v * erfcf(v * -0.70710678118654752440f);
}
__device__ __forceinline__ float gelu_slope_f32(float v) {
  const float a = v < -24.f ? -24.f : v > 24.f ? 24.f : v;
  return fmaf(0.39894228040143267794f * a, expf(-0.5f * a * a), 0.5f * erfcf(a * -0.70710678118654752440f));
}

}  // namespace vit
