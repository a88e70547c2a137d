// Queries and keys behind a projection: norm of each head and rotation of its leading entries by the row's position, in one pass.
//
//   z = x / sqrt(mean x^2 + eps) * w          or   (x - mean) / sqrt(var + eps) * w + b          (head of D entries)
//   (u, v) -> (u cos t - v sin t, v cos t + u sin t),   t = pos[axis of the pair] * frequency of the pair
//
// Angles.  A frequency is kept as a 64-bit fraction of a turn, F = 2^64 frac(f / 2 pi); pos * F modulo 2^64 is the exact fraction of a
// turn that the rounded F gives at an int32 position: off by 2^31 * 2^-65 turns (4e-10 radians) at most.  It is rounded to 32 bits (7e-10
// radians), the nearest quarter turn is taken off in integers and only the rest, at most an eighth of a turn, becomes a float: three
// roundings of 2^-24 of it, 1.4e-7 radians at an eighth of a turn.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "lq_device.cuh"
#include "lq_heads_cut.h"
#include "lq_heads_places.h"
#include "lq_internal.h"
#include "lq_turns.h"

using namespace lqdev;

namespace {

constexpr int MAX_D = 256, WARPS = LQ_HEADS_WARPS, MAX_ROWS = LQ_HEADS_ROWS;
enum { ROT_NONE = 0, ROT_PAIRS = 1, ROT_HALVES = 2 };

struct Side {
  const void* in;
  void* out;
  int in_seq, in_row, in_head, out_seq, out_row, out_head;
  const float *weight, *bias;
};
struct HeadsParams {
  Side side[2];
  int rows, heads[2], seq_len, lanes, groups, axes, pairs;
  int block_rows, walk, parts[2];   // rows of a block; heads a warp walks over at a time, and the parts that makes of Q's and K's
  uint32_t by_parts, by_wide, by_groups;   // 2^32 / divisor, rounded up, of parts[0] + parts[1], of the pairs rounded up to four, of groups:
                                // quotients of what is below 2^16 (a divisor of one is not divided by)
  float eps, inv_d;
  const uint64_t* turn;
  const uint8_t* axis;
  const int32_t* pos;
};

// eight entries: two runs of four neighbours, `apart` entries from the first to the second (4: one run of eight)
template <typename T> struct Raw;
template <> struct Raw<__half> { uint2 a, b; };
template <> struct Raw<float> { float4 a, b; };
template <bool SPLIT>
__device__ __forceinline__ Raw<__half> load_raw(const __half* p, int apart) {
  if constexpr (SPLIT) return {*reinterpret_cast<const uint2*>(p), *reinterpret_cast<const uint2*>(p + apart)};
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  return {make_uint2(v.x, v.y), make_uint2(v.z, v.w)};
}
template <bool SPLIT>
__device__ __forceinline__ Raw<float> load_raw(const float* p, int apart) {
  return {*reinterpret_cast<const float4*>(p), *reinterpret_cast<const float4*>(p + (SPLIT ? apart : 4))};
}
// The four pairs of a lane: first sides lo, second sides hi, two pairs to a register pair (packed arithmetic takes both at once).
// NEIGHBOURS: a pair is two neighbouring entries.
struct Pairs {
  float2 lo[2], hi[2];
};
template <bool NEIGHBOURS>
__device__ __forceinline__ Pairs open8(const Raw<float>& r) {
  if constexpr (NEIGHBOURS)
    return {{make_float2(r.a.x, r.a.z), make_float2(r.b.x, r.b.z)}, {make_float2(r.a.y, r.a.w), make_float2(r.b.y, r.b.w)}};
  return {{make_float2(r.a.x, r.a.y), make_float2(r.a.z, r.a.w)}, {make_float2(r.b.x, r.b.y), make_float2(r.b.z, r.b.w)}};
}
template <bool NEIGHBOURS>
__device__ __forceinline__ Pairs open8(const Raw<__half>& r) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.b.x, r.b.y};
  float2 f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
  return open8<NEIGHBOURS>(Raw<float>{make_float4(f[0].x, f[0].y, f[1].x, f[1].y), make_float4(f[2].x, f[2].y, f[3].x, f[3].y)});
}
template <bool NEIGHBOURS>
__device__ __forceinline__ Raw<float> close8(const Pairs& x) {
  if constexpr (NEIGHBOURS)
    return {make_float4(x.lo[0].x, x.hi[0].x, x.lo[0].y, x.hi[0].y), make_float4(x.lo[1].x, x.hi[1].x, x.lo[1].y, x.hi[1].y)};
  return {make_float4(x.lo[0].x, x.lo[0].y, x.lo[1].x, x.lo[1].y), make_float4(x.hi[0].x, x.hi[0].y, x.hi[1].x, x.hi[1].y)};
}
template <bool SPLIT>
__device__ __forceinline__ void store_raw(float* p, int apart, const Raw<float>& x) {
  *reinterpret_cast<float4*>(p) = x.a;
  *reinterpret_cast<float4*>(p + (SPLIT ? apart : 4)) = x.b;
}
template <bool SPLIT>
__device__ __forceinline__ void store_raw(__half* p, int apart, const Raw<float>& x) {
  const __half2 h[4] = {__floats2half2_rn(x.a.x, x.a.y), __floats2half2_rn(x.a.z, x.a.w), __floats2half2_rn(x.b.x, x.b.y), __floats2half2_rn(x.b.z, x.b.w)};
  const uint4 v = *reinterpret_cast<const uint4*>(h);
  if constexpr (SPLIT) {
    *reinterpret_cast<uint2*>(p) = make_uint2(v.x, v.y);
    *reinterpret_cast<uint2*>(p + apart) = make_uint2(v.z, v.w);
  } else {
    *reinterpret_cast<uint4*>(p) = v;
  }
}
__device__ __forceinline__ float2 both(float a) { return make_float2(a, a); }

// Cosine and sine of pos * turn.  Taylor's series about the nearest quarter turn, at most pi / 4 away: the terms left out are below 2e-9 and 2e-10.
__device__ __forceinline__ float2 cos_sin(uint64_t turn, int32_t pos) {
  const int32_t t = (int32_t)(uint32_t)((turn * (uint64_t)(int64_t)pos + 0x80000000u) >> 32);       // fraction of a turn, 2^32 = 1
  const uint32_t quarter = ((uint32_t)t + 0x20000000u) >> 30;                          // nearest quarter turn, 0 .. 3
  const int32_t rest = (int32_t)((uint32_t)t - (quarter << 30));                       // [-2^29, 2^29)
  const float x = (float)rest * 1.46291807926715968e-9f, y = x * x;                    // 2 pi / 2^32
  float s = fmaf(y, 2.75573192239858907e-6f, -1.98412698412698413e-4f);
  s = fmaf(s, y, 8.33333333333333333e-3f);
  s = fmaf(s, y, -1.66666666666666667e-1f);
  s = fmaf(s * y, x, x);
  float c = fmaf(y, -2.75573192239858907e-7f, 2.48015873015873016e-5f);
  c = fmaf(c, y, -1.38888888888888889e-3f);
  c = fmaf(c, y, 4.16666666666666667e-2f);
  c = fmaf(c, y, -0.5f);
  c = fmaf(c, y, 1.f);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;                        // one quarter on: (-s, c)
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

// Sum over a group's L neighbouring lanes, in every lane of it.  Powers of two: xor steps.  Other L known at compile time: sums over windows of
// 1, .., L lanes round the group, each twice the one before or one longer (L = 9: 1, 2, 4, 8, 9).  L = 0: `lanes` lanes, summed up to the group's
// first lane and handed back.
template <int L>
__device__ __forceinline__ float group_sum(float a, int lanes, int at, int lane) {
  if constexpr (L > 0 && (L & (L - 1)) == 0) {
#pragma unroll
    for (int d = L / 2; d > 0; d /= 2) a += __shfl_xor_sync(0xffffffffu, a, d);
  } else if constexpr (L > 0) {
    const float one = a;
    int len = 1;
#pragma unroll
    for (int bit = L >= 16 ? 3 : L >= 8 ? 2 : L >= 4 ? 1 : 0; bit >= 0; --bit) {
      a += __shfl_sync(0xffffffffu, a, lane + (at + len >= L ? len - L : len));
      len *= 2;
      if ((L >> bit) & 1) {
        a += __shfl_sync(0xffffffffu, one, lane + (at + len >= L ? len - L : len));
        ++len;
      }
    }
  } else {
#pragma unroll
    for (int d = 1; d < 32; d *= 2)
      if (d < lanes) {
        const float u = __shfl_down_sync(0xffffffffu, a, d);
        if (at + d < lanes) a += u;
      }
    a = __shfl_sync(0xffffffffu, a, lane - at);
  }
  return a;
}

// A block takes a few rows and forms their angles together.  Its warps share out the rows' heads: one walks over the queries, or the keys, of
// a row, or over a part of them.  L lanes hold a head, each lane C times eight entries that are the two sides of the same four pairs in every
// head, so weights times cosines and sines stay in registers along the walk; the norm's sum crosses the head's lanes by shuffles.  What
// bounds it short of the memory is the issue of instructions (32 heads of 72: 1924 a row at first, 64-bit address arithmetic and moves most
// of them) and warps enough to cover their latency: where L is known (then the whole head is rotated, or nothing) every address is a base and
// a constant; a lane holds 16 entries of heads of 64 and 128, but of 72 only 8 (24, for three lanes a head, take 128 registers: 24.7 us for
// 18.9); blocks are small, so that few warps wait for the angles of others.  (The bounds of 72 and 96 registers cost up to 20 bytes of spills in
// the fp16 instances.)
// B200, us in a graph of ten passes and share of the measured copy rate of its bytes: 32760 rows, 40 heads of 128, fp16 110.6, 0.93 (in long runs
// 116 to 118, 0.87); 8192 rows, 32 heads of 72, fp16 19.0, 0.61; 4100 rows, 32 heads of 128, fp32, no norm 24.7, 0.83; one row 2.1.
template <typename TIN, typename TOUT, int NORM, int ROT, int L, int C>
__global__ void __launch_bounds__(32 * WARPS, C == 1 && sizeof(TIN) == 2 && NORM != LQ_NORM_LAYER ? 7 : C == 2 && sizeof(TIN) == 2 ? 5 : 4)
    lq_heads_kernel(const __grid_constant__ HeadsParams p) {
  constexpr bool SPLIT = ROT == ROT_HALVES, NEIGHBOURS = ROT == ROT_PAIRS, FIXED = L > 0;
  static_assert(FIXED || C == 1, "");
  constexpr int DEPTH = sizeof(TIN) == 2 ? 3 : C == 1 ? 3 : 2;      // heads of a lane in flight
  constexpr int UNIT = SPLIT ? 4 : 8;                     // entries from one lane's to the next one's
  __shared__ __align__(16) float trig[ROT == ROT_NONE ? 1 : MAX_ROWS * MAX_D];         // [rows of the block][cos, sin][pairs, a multiple of four]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, lanes = FIXED ? L : p.lanes, groups = FIXED ? 32 / (FIXED ? L : 1) : p.groups;
  int grp = 0;
  if constexpr (FIXED) grp = lane / L;
  else
    for (int i = lanes; i <= lane; i += lanes) ++grp;
  const int v = lane - grp * lanes;
  const bool works = (FIXED && 32 % (FIXED ? L : 1) == 0) || grp < groups;
  const int row0 = blockIdx.x * p.block_rows, wide = (p.pairs + 3) & ~3, parts = p.parts[0] + p.parts[1];
  const int tasks = min(p.block_rows, p.rows - row0) * parts;
  const int seq0 = row0 / p.seq_len, at0 = row0 - seq0 * p.seq_len;
  // pairs 4 i .. 4 i + 3 of the lane's i = v, v + L, ..: entries 8 i .. 8 i + 7, or (halves) 4 i .. 4 i + 3 and as many half of the rotated part
  // further; what is not rotated lies behind, eight neighbours at a time
  const int turns = ROT == ROT_NONE ? 0 : FIXED ? 4 : max(0, min(4, p.pairs - 4 * v));        // pairs that are rotated
  const int first = FIXED || turns > 0 ? UNIT * v : 8 * v, apart = !SPLIT ? 4 : FIXED ? 4 * L * C : turns > 0 ? p.pairs : 4;
  grid_launch_dependents();
  grid_dependency_wait();
  int task = blockIdx.y * WARPS + warp, r = 0, which = 0, begin = 0, end = 0, left = 0, in_step = 0, out_step = 0;
  const TIN* in = nullptr;
  TOUT* out = nullptr;
  Raw<TIN> raw[DEPTH][C];                                 // (what is not loaded is computed with and not stored)
  const auto open_task = [&]() {                          // where the task's heads lie; the first ones are asked for
    r = parts == 1 ? task : (int)__umulhi(task, p.by_parts);
    const int part = task - r * parts;
    which = part >= p.parts[0];
    const Side& side = p.side[which];
    begin = (part - (which ? p.parts[0] : 0)) * p.walk;
    end = min(p.heads[which], begin + p.walk);
    int seq = seq0, at = at0 + r;
    for (; at >= p.seq_len; at -= p.seq_len) ++seq;
    in_step = groups * side.in_head; out_step = groups * side.out_head;
    in = reinterpret_cast<const TIN*>(side.in) +
         ((long long)seq * side.in_seq + (long long)at * side.in_row + (long long)(begin + grp) * side.in_head + first);
    out = reinterpret_cast<TOUT*>(side.out) +
          ((long long)seq * side.out_seq + (long long)at * side.out_row + (long long)(begin + grp) * side.out_head + first);
    left = works ? end - begin - grp : 0;                 // heads that this lane has before it, in steps of `groups`
#pragma unroll
    for (int u = 0; u < DEPTH; ++u) {
      if (left > u * groups)
#pragma unroll
        for (int i = 0; i < C; ++i) raw[u][i] = load_raw<SPLIT>(in + UNIT * L * i, apart);
      in += in_step;
    }
  };
  if (task < tasks) open_task();
  if constexpr (ROT != ROT_NONE) {
    for (int e = threadIdx.x; e < wide * p.block_rows; e += 32 * WARPS) {
      const int r = (int)__umulhi(e, p.by_wide), i = e - r * wide;
      float2 cs = make_float2(1.f, 0.f);                  // (pairs behind the rotated ones stay)
      if (i < p.pairs && row0 + r < p.rows) cs = cos_sin(p.turn[i], p.pos[(long long)(row0 + r) * p.axes + p.axis[i]]);
      trig[2 * r * wide + i] = cs.x;
      trig[(2 * r + 1) * wide + i] = cs.y;
    }
    __syncthreads();
  }
#pragma unroll 1
  while (task < tasks) {
    const Side& side = p.side[which];
    Pairs w[C], cross[C], b[NORM == LQ_NORM_LAYER ? C : 1];       // cross: lo is hi's share in lo, hi is lo's share in hi
#pragma unroll
    for (int i = 0; i < C; ++i) {
      w[i] = {{both(1.f), both(1.f)}, {both(1.f), both(1.f)}};
      if constexpr (NORM != LQ_NORM_NONE)
        if (works && side.weight) w[i] = open8<NEIGHBOURS>(load_raw<SPLIT>(side.weight + first + UNIT * L * i, apart));
      if constexpr (NORM == LQ_NORM_LAYER) {
        b[i] = {};
        if (works && side.bias) b[i] = open8<NEIGHBOURS>(load_raw<SPLIT>(side.bias + first + UNIT * L * i, apart));
      }
      if (ROT != ROT_NONE && turns > 0) {
        const float* t = trig + 2 * r * wide + 4 * (v + i * L);
        const float4 c4 = *reinterpret_cast<const float4*>(t), s4 = *reinterpret_cast<const float4*>(t + wide);
        const float2 c[2] = {make_float2(c4.x, c4.y), make_float2(c4.z, c4.w)}, s[2] = {make_float2(s4.x, s4.y), make_float2(s4.z, s4.w)};
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const float2 neg = make_float2(-s[q].x, -s[q].y);
          cross[i].lo[q] = __fmul2_rn(w[i].hi[q], neg);
          cross[i].hi[q] = __fmul2_rn(w[i].lo[q], s[q]);
          w[i].lo[q] = __fmul2_rn(w[i].lo[q], c[q]);
          w[i].hi[q] = __fmul2_rn(w[i].hi[q], c[q]);
          if constexpr (NORM == LQ_NORM_LAYER) {
            const float2 l = b[i].lo[q];
            b[i].lo[q] = __ffma2_rn(b[i].hi[q], neg, __fmul2_rn(l, c[q]));
            b[i].hi[q] = __ffma2_rn(l, s[q], __fmul2_rn(b[i].hi[q], c[q]));
          }
        }
      }
    }
    int steps = groups == 1 ? end - begin : (int)__umulhi(end - begin + groups - 1, p.by_groups);
#pragma unroll 1
    while (steps > 0) {
#pragma unroll
      for (int u = 0; u < DEPTH; ++u) {
        if (u > 0 && steps <= 0) break;
        Pairs x[C];
#pragma unroll
        for (int i = 0; i < C; ++i) x[i] = open8<NEIGHBOURS>(raw[u][i]);
        if (left > DEPTH * groups)
#pragma unroll
          for (int i = 0; i < C; ++i) raw[u][i] = load_raw<SPLIT>(in + UNIT * L * i, apart);
        float2 scale = both(1.f);
        if constexpr (NORM == LQ_NORM_LAYER) {
          float2 t = both(0.f);
#pragma unroll
          for (int i = 0; i < C; ++i) t = __fadd2_rn(t, __fadd2_rn(__fadd2_rn(x[i].lo[0], x[i].lo[1]), __fadd2_rn(x[i].hi[0], x[i].hi[1])));
          const float2 m = both(-group_sum<L>(t.x + t.y, lanes, v, lane) * p.inv_d);
#pragma unroll
          for (int i = 0; i < C; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q) { x[i].lo[q] = __fadd2_rn(x[i].lo[q], m); x[i].hi[q] = __fadd2_rn(x[i].hi[q], m); }
        }
        if constexpr (NORM != LQ_NORM_NONE) {
          float2 t[2] = {both(0.f), both(0.f)};
#pragma unroll
          for (int i = 0; i < C; ++i)
#pragma unroll
            for (int q = 0; q < 2; ++q) t[q] = __ffma2_rn(x[i].hi[q], x[i].hi[q], __ffma2_rn(x[i].lo[q], x[i].lo[q], t[q]));
          const float2 a = __fadd2_rn(t[0], t[1]);
          scale = both(rsqrtf(fmaf(group_sum<L>(a.x + a.y, lanes, v, lane), p.inv_d, p.eps)));
        }
#pragma unroll
        for (int i = 0; i < C; ++i) {
          Pairs y;
#pragma unroll
          for (int q = 0; q < 2; ++q) { y.lo[q] = __fmul2_rn(x[i].lo[q], w[i].lo[q]); y.hi[q] = __fmul2_rn(x[i].hi[q], w[i].hi[q]); }
          if constexpr (ROT != ROT_NONE && FIXED) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              y.lo[q] = __ffma2_rn(x[i].hi[q], cross[i].lo[q], y.lo[q]);
              y.hi[q] = __ffma2_rn(x[i].lo[q], cross[i].hi[q], y.hi[q]);
            }
          } else if constexpr (ROT != ROT_NONE) {         // (an infinity that is not rotated stays where it is)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              if (2 * q < turns) {
                y.lo[q].x = fmaf(x[i].hi[q].x, cross[i].lo[q].x, y.lo[q].x);
                y.hi[q].x = fmaf(x[i].lo[q].x, cross[i].hi[q].x, y.hi[q].x);
              }
              if (2 * q + 1 < turns) {
                y.lo[q].y = fmaf(x[i].hi[q].y, cross[i].lo[q].y, y.lo[q].y);
                y.hi[q].y = fmaf(x[i].lo[q].y, cross[i].hi[q].y, y.hi[q].y);
              }
            }
          }
          if constexpr (NORM != LQ_NORM_NONE) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              y.lo[q] = NORM == LQ_NORM_LAYER ? __ffma2_rn(y.lo[q], scale, b[i].lo[q]) : __fmul2_rn(y.lo[q], scale);
              y.hi[q] = NORM == LQ_NORM_LAYER ? __ffma2_rn(y.hi[q], scale, b[i].hi[q]) : __fmul2_rn(y.hi[q], scale);
            }
          }
          if (left > 0) store_raw<SPLIT>(out + UNIT * L * i, apart, close8<NEIGHBOURS>(y));
        }
        in += in_step;
        out += out_step;
        left -= groups;
        --steps;
      }
    }
    task += WARPS * gridDim.y;
    if (task < tasks) open_task();
  }
}

template <typename TIN, typename TOUT, int NORM, int ROT, int L, int C>
cudaError_t launch(HeadsParams& p, int sms, cudaStream_t st) {
  p.lanes = L > 0 ? L : p.lanes;
  p.groups = 32 / p.lanes;
  const int g = p.groups;
  const LqHeadsCut c = lq_heads_cut(p.rows, p.heads[0], p.heads[1], g, sms);
  p.walk = c.walk;
  p.block_rows = c.block_rows;
  for (int i = 0; i < 2; ++i) p.parts[i] = c.parts[i];
  const auto reciprocal = [](int d) { return (uint32_t)(((1ull << 32) + d - 1) / d); };
  p.by_parts = reciprocal(std::max(2, c.parts[0] + c.parts[1]));
  p.by_wide = reciprocal(std::max(4, lq_round_up(p.pairs, 4)));
  p.by_groups = reciprocal(std::max(2, g));
  return lq_launch_grid(lq_heads_kernel<TIN, TOUT, NORM, ROT, L, C>, dim3(c.blocks, c.blocks_y), 32 * WARPS, 1, 0, st, p);
}
// Under an RMS norm heads of 64, 72, 112 and 128 entries that are rotated as a whole, or not at all, have their lanes at compile time, 16
// entries to each where lanes are a power of two; others hold eight entries a lane.  us of 8192 rows of 32 heads by these and by the general
// form: fp16, rotated 64 16.5 / 18.6, 72 18.8 / 24.3, 112 25.0 / 29.8, 128 25.5 / 30.1; fp16, not rotated 13.9 / 14.9, 16.8 / 19.2, 22.4 / 24.6,
// 22.9 / 25.3; fp32, rotated 25.3 / 29.6, 34.6 / 39.1, 46.9 / 50.9, 42.5 / 52.5; of 64 rows 2.3 to 2.5 / 2.5 to 2.8.
template <typename TIN, typename TOUT, int NORM, int ROT>
cudaError_t launch_lanes(HeadsParams& p, int sms, cudaStream_t st) {
  if constexpr (NORM == LQ_NORM_RMS)
    if (ROT == ROT_NONE || p.pairs == 4 * p.lanes) {
      if (p.lanes == 8) return launch<TIN, TOUT, NORM, ROT, 4, 2>(p, sms, st);
      if (p.lanes == 9) return launch<TIN, TOUT, NORM, ROT, 9, 1>(p, sms, st);
      if (p.lanes == 14) return launch<TIN, TOUT, NORM, ROT, 14, 1>(p, sms, st);
      if (p.lanes == 16) return launch<TIN, TOUT, NORM, ROT, 8, 2>(p, sms, st);
    }
  return launch<TIN, TOUT, NORM, ROT, 0, 1>(p, sms, st);
}
template <typename TIN, typename TOUT, int NORM>
cudaError_t launch_rot(HeadsParams& p, int rot, int sms, cudaStream_t st) {
  return rot == ROT_NONE    ? launch_lanes<TIN, TOUT, NORM, ROT_NONE>(p, sms, st)
         : rot == ROT_PAIRS ? launch_lanes<TIN, TOUT, NORM, ROT_PAIRS>(p, sms, st)
                            : launch_lanes<TIN, TOUT, NORM, ROT_HALVES>(p, sms, st);
}
template <typename TIN, typename TOUT>
cudaError_t launch_norm(HeadsParams& p, int norm, int rot, int sms, cudaStream_t st) {
  return norm == LQ_NORM_NONE  ? launch_rot<TIN, TOUT, LQ_NORM_NONE>(p, rot, sms, st)
         : norm == LQ_NORM_RMS ? launch_rot<TIN, TOUT, LQ_NORM_RMS>(p, rot, sms, st)
                               : launch_rot<TIN, TOUT, LQ_NORM_LAYER>(p, rot, sms, st);
}

// Strides over dimensions of one entry mean nothing; the others keep entries on 16-byte boundaries.
lq_status take_side(const lq_heads* h, int sequences, int seq_len, lq_norm norm, bool same_type, Side* s) {
  if (!h->in || !h->out || h->heads < 1) return LQ_ERR_INVALID_ARG;
  if (h->heads > 4096) return LQ_ERR_UNSUPPORTED;
  if ((((uintptr_t)h->in | (uintptr_t)h->out | (uintptr_t)h->weight | (uintptr_t)h->bias) & 15) != 0) return LQ_ERR_INVALID_ARG;
  if ((h->weight && norm == LQ_NORM_NONE) || (h->bias && norm != LQ_NORM_LAYER)) return LQ_ERR_INVALID_ARG;
  const int64_t strides[6] = {sequences == 1 ? 0 : h->in_seq, seq_len == 1 ? 0 : h->in_row, h->heads == 1 ? 0 : h->in_head,
                              sequences == 1 ? 0 : h->out_seq, seq_len == 1 ? 0 : h->out_row, h->heads == 1 ? 0 : h->out_head};
  for (int64_t v : strides) {
    if (v % 8 != 0) return LQ_ERR_INVALID_ARG;
    if (v > INT32_MAX || v < -INT32_MAX) return LQ_ERR_UNSUPPORTED;
  }
  for (int i : {2, 5})                                       // (a warp steps over up to 32 heads)
    if (strides[i] > INT32_MAX / 32 || strides[i] < -(INT32_MAX / 32)) return LQ_ERR_UNSUPPORTED;
  *s = Side{h->in, h->out, (int)strides[0], (int)strides[1], (int)strides[2], (int)strides[3], (int)strides[4], (int)strides[5], h->weight, h->bias};
  if (h->in == h->out && (!same_type || strides[0] != strides[3] || strides[1] != strides[4] || strides[2] != strides[5])) return LQ_ERR_INVALID_ARG;
  return LQ_OK;
}

// No two outputs on one place, and none on an input, but for a side that is worked on in place (in == out: the same strides and type by now).
lq_status check_places(const HeadsParams& p, int head_dim, int sequences, lq_out_dtype in_dtype, lq_out_dtype out_dtype) {
  const auto runs = [&](const void* at, int seq, int row, int head, int heads, lq_out_dtype dt) {
    const int64_t esz = dt == LQ_OUT_F32 ? 4 : 2;
    return LqRuns{(uintptr_t)at, {seq * esz, row * esz, head * esz}, {sequences, p.seq_len, heads}, head_dim * esz};
  };
  const auto line = [](const void* at, int64_t bytes) { return LqRuns{(uintptr_t)at, {0, 0, 0}, {1, 1, 1}, bytes}; };
  LqRuns out[2], in[9];                                      // in: of both sides, their weights and biases, the positions
  int n_out = 0, n_in = 0;
  for (int i = 0; i < 2; ++i) {
    if (p.heads[i] == 0) continue;
    const Side& s = p.side[i];
    out[n_out++] = runs(s.out, s.out_seq, s.out_row, s.out_head, p.heads[i], out_dtype);
    if (s.in != s.out) in[n_in++] = runs(s.in, s.in_seq, s.in_row, s.in_head, p.heads[i], in_dtype);
    if (s.weight) in[n_in++] = line(s.weight, head_dim * 4);
    if (s.bias) in[n_in++] = line(s.bias, head_dim * 4);
  }
  if (p.pairs > 0) in[n_in++] = line(p.pos, (int64_t)p.rows * p.axes * 4);
  const auto status = [](LqPlaces c) { return c == LQ_APART ? LQ_OK : c == LQ_SHARED ? LQ_ERR_INVALID_ARG : LQ_ERR_UNSUPPORTED; };
  lq_status s = n_out > 1 ? status(lq_runs_meet(out[0], out[1])) : LQ_OK;
  for (int i = 0; i < n_out && s == LQ_OK; ++i) {
    s = status(lq_runs_collide(out[i]));
    for (int j = 0; j < n_in && s == LQ_OK; ++j) s = status(lq_runs_meet(out[i], in[j]));
  }
  return s;
}

}  // namespace

extern "C" lq_status lq_rope_config_default(lq_rope_config* cfg, int32_t axes, const int32_t* dims) {
  if (!cfg || axes < 0 || axes > LQ_ROPE_MAX_AXES || (axes > 0 && !dims)) return LQ_ERR_INVALID_ARG;
  *cfg = lq_rope_config{};
  cfg->axes = axes;
  for (int a = 0; a < axes; ++a) cfg->dims[a] = dims[a];
  cfg->theta = 10000.0;
  return LQ_OK;
}

extern "C" lq_status lq_rope_create(const lq_rope_config* cfg, const double* freq, const int32_t* axis, int device, lq_rope** out) {
  if (!cfg || !out || cfg->axes < 0 || cfg->axes > LQ_ROPE_MAX_AXES) return LQ_ERR_INVALID_ARG;
  if ((cfg->halves != 0 && cfg->halves != 1) || (cfg->shared != 0 && cfg->shared != 1)) return LQ_ERR_INVALID_ARG;
  if (!(cfg->theta > 0) || !isfinite(cfg->theta)) return LQ_ERR_INVALID_ARG;
  int rot = 0;
  for (int a = 0; a < cfg->axes; ++a) {
    if (cfg->dims[a] < 0 || cfg->dims[a] % 2 != 0) return LQ_ERR_INVALID_ARG;
    if (cfg->dims[a] > MAX_D || (rot += cfg->dims[a]) > MAX_D) return LQ_ERR_UNSUPPORTED;
  }
  if (cfg->halves && rot % 8 != 0) return LQ_ERR_UNSUPPORTED;
  std::vector<uint64_t> turn;
  std::vector<uint8_t> which;
  try {
    turn.reserve(MAX_D / 2); which.reserve(MAX_D / 2);
    int i = 0;
    for (int a = 0; a < cfg->axes; ++a)
      for (int j = 0; j < cfg->dims[a] / 2; ++j, ++i) {
        if (axis && (axis[i] < 0 || axis[i] >= cfg->axes)) return LQ_ERR_INVALID_ARG;
        const long double f = freq ? (long double)freq[i]
                                   : powl((long double)cfg->theta, -2.0L * (cfg->shared ? i : j) / (cfg->shared ? rot : cfg->dims[a]));
        if (!isfinite(f)) return LQ_ERR_NUMERIC;
        if (fabsl(f) >= 0x1p64L) return LQ_ERR_UNSUPPORTED;
        turn.push_back(lq_turn_fraction(f));
        which.push_back((uint8_t)(axis ? axis[i] : a));
      }
  } catch (const std::bad_alloc&) { return LQ_ERR_ALLOC; }
  int ndev = 0;
  if (lq_note_cuda(cudaGetDeviceCount(&ndev)) != cudaSuccess || device < 0 || device >= ndev) return LQ_ERR_CUDA;
  LqDeviceGuard guard(device);
  if (!guard.ok) return LQ_ERR_CUDA;
  lq_rope* R = new (std::nothrow) lq_rope{cfg->axes, rot / 2, cfg->halves, device, 0, nullptr, nullptr};
  if (!R) return LQ_ERR_ALLOC;
  if (lq_note_cuda(cudaDeviceGetAttribute(&R->sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) {
    lq_rope_free(R);
    return LQ_ERR_CUDA;
  }
  if (rot > 0) {
    const size_t n = turn.size();
    if (lq_note_cuda(cudaMalloc((void**)&R->d_turn, n * sizeof(uint64_t))) != cudaSuccess ||
        lq_note_cuda(cudaMalloc((void**)&R->d_axis, n)) != cudaSuccess) {
      lq_rope_free(R);
      return LQ_ERR_ALLOC;
    }
    if (lq_note_cuda(cudaMemcpy(R->d_turn, turn.data(), n * sizeof(uint64_t), cudaMemcpyHostToDevice)) != cudaSuccess ||
        lq_note_cuda(cudaMemcpy(R->d_axis, which.data(), n, cudaMemcpyHostToDevice)) != cudaSuccess ||
        lq_note_cuda(cudaDeviceSynchronize()) != cudaSuccess) {
      lq_rope_free(R);
      return LQ_ERR_CUDA;
    }
  }
  *out = R;
  return LQ_OK;
}

extern "C" lq_status lq_rope_free(lq_rope* R) {
  if (!R) return LQ_ERR_INVALID_ARG;
  LqDeviceGuard guard(R->device);
  cudaFree(R->d_turn); cudaFree(R->d_axis);
  delete R;
  return LQ_OK;
}

lq_status lq_heads_run(const lq_heads* q, const lq_heads* k, int32_t head_dim, int32_t sequences, int32_t seq_len, lq_norm norm, float eps, const lq_rope* R,
                       const int32_t* pos, lq_out_dtype in_dtype, lq_out_dtype out_dtype, int device, bool launch, cudaStream_t st) {
  if (!R || (!q && !k) || sequences < 1 || seq_len < 1 || head_dim < 1) return LQ_ERR_INVALID_ARG;
  if (norm != LQ_NORM_NONE && norm != LQ_NORM_RMS && norm != LQ_NORM_LAYER) return LQ_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !isfinite(eps)) return LQ_ERR_INVALID_ARG;
  for (lq_out_dtype d : {in_dtype, out_dtype})
    if (d != LQ_OUT_F16 && d != LQ_OUT_F32) return LQ_ERR_INVALID_ARG;
  if (head_dim % 8 != 0 || head_dim > MAX_D) return LQ_ERR_UNSUPPORTED;
  if (2 * R->pairs > head_dim || (R->pairs > 0 && (!pos || ((uintptr_t)pos & 3) != 0))) return LQ_ERR_INVALID_ARG;
  const long long rows = (long long)sequences * seq_len;
  if (rows > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  HeadsParams p = {};
  lq_status s;
  const lq_heads* both[2] = {q, k};
  for (int i = 0; i < 2; ++i)
    if (both[i] && (s = take_side(both[i], sequences, seq_len, norm, in_dtype == out_dtype, &p.side[i])) != LQ_OK) return s;
  p.heads[0] = q ? q->heads : 0;
  p.heads[1] = k ? k->heads : 0;
  p.rows = (int)rows;
  p.lanes = head_dim / 8;
  p.seq_len = seq_len; p.axes = R->axes; p.pairs = R->pairs;
  p.eps = eps; p.inv_d = 1.f / (float)head_dim;
  p.turn = R->d_turn; p.axis = R->d_axis; p.pos = pos;
  if (device >= 0 && device != R->device) return LQ_ERR_INVALID_ARG;
  if ((s = check_places(p, head_dim, sequences, in_dtype, out_dtype)) != LQ_OK || !launch) return s;
  LqDeviceGuard guard(R->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  const int rot = R->pairs == 0 ? ROT_NONE : R->halves ? ROT_HALVES : ROT_PAIRS, sms = R->sms;
  const bool f32_out = out_dtype == LQ_OUT_F32;
  const cudaError_t e =
      in_dtype == LQ_OUT_F16 ? (f32_out ? launch_norm<__half, float>(p, norm, rot, sms, st) : launch_norm<__half, __half>(p, norm, rot, sms, st))
                             : (f32_out ? launch_norm<float, float>(p, norm, rot, sms, st) : launch_norm<float, __half>(p, norm, rot, sms, st));
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}

extern "C" lq_status lq_qk_norm_rope(const lq_heads* q, const lq_heads* k, int32_t head_dim, int32_t sequences, int32_t seq_len, lq_norm norm,
                                     float eps, const lq_rope* R, const int32_t* pos, lq_out_dtype in_dtype, lq_out_dtype out_dtype, void* stream) {
  return lq_heads_run(q, k, head_dim, sequences, seq_len, norm, eps, R, pos, in_dtype, out_dtype, -1, true, (cudaStream_t)stream);
}
