// The residual stream between two blocks, in one pass over its rows:
//
//   x' = x + factor * gate * N1(y),   h = (N2(x') * w + b) * (1 + scale) + shift
//
// N: none, RMS or LayerNorm of a row; gate, scale and shift are a sequence's.  Reads x and y once and writes x' and h once; the memory
// bounds it.  A row is held in registers by one to eight warps, up to nine times four neighbouring entries a lane, all asked for at once and
// kept as they lie in memory until they are used, so that many rows are on their way.  What a row is multiplied with and what is added is
// put together once for a sequence's rows of a thread block, in shared memory, and arithmetic goes two entries at a time: with five vectors
// from global memory a row and entry by entry the issue of instructions took most of the time (32768 rows of 2240, fp32 stream: 369 us; now
// 151 us, 5.8 TB/s, 0.89 of the measured copy rate, after a pause, and 154 back to back).
// Variances are sums about the mean that is known; h is made of x' before that is rounded to its type.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "lq_device.cuh"
#include "lq_heads_places.h"
#include "lq_internal.h"

using namespace lqdev;

namespace {

constexpr int THREADS = 256, WARPS = THREADS / 32;

struct ResidualParams {
  const void *x, *y;
  void *x_out, *h;
  long long x_row, y_row, x_out_row, h_row, mod_seq;
  const float *after_weight, *weight, *bias;
  const void *gate, *scale, *shift;
  int rows, features, seq_rows, after, norm, mod_f32, wide;            // seq_rows: rows that have the same vectors; wide: warps of a row
  int groups, seq_groups, share;         // groups of rows that a thread block takes at once, of all rows and of a sequence; groups a block takes
  float factor, eps, inv;
};

struct Four {
  float2 lo, hi;
};
template <bool F32> struct Raw;
template <> struct Raw<false> {
  uint2 a;
  __device__ __forceinline__ static Raw load(const uint8_t* p) { return {*reinterpret_cast<const uint2*>(p)}; }
  __device__ __forceinline__ static Raw zero() { return {make_uint2(0, 0)}; }
  __device__ __forceinline__ Four open() const {
    return {__half22float2(*reinterpret_cast<const __half2*>(&a.x)), __half22float2(*reinterpret_cast<const __half2*>(&a.y))};
  }
  __device__ __forceinline__ static void store(uint8_t* p, const Four& e) {
    const __half2 a = __floats2half2_rn(e.lo.x, e.lo.y), b = __floats2half2_rn(e.hi.x, e.hi.y);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
};
template <> struct Raw<true> {
  float4 a;
  __device__ __forceinline__ static Raw load(const uint8_t* p) { return {*reinterpret_cast<const float4*>(p)}; }
  __device__ __forceinline__ static Raw zero() { return {make_float4(0.f, 0.f, 0.f, 0.f)}; }
  __device__ __forceinline__ Four open() const { return {make_float2(a.x, a.y), make_float2(a.z, a.w)}; }
  __device__ __forceinline__ static void store(uint8_t* p, const Four& e) { *reinterpret_cast<float4*>(p) = make_float4(e.lo.x, e.lo.y, e.hi.x, e.hi.y); }
};
__device__ __forceinline__ Four load4(const void* p, long long at, bool f32) {
  return f32 ? Raw<true>::load(reinterpret_cast<const uint8_t*>(p) + 4 * at).open() : Raw<false>::load(reinterpret_cast<const uint8_t*>(p) + 2 * at).open();
}
__device__ __forceinline__ Four mul(const Four& a, const Four& b) { return {__fmul2_rn(a.lo, b.lo), __fmul2_rn(a.hi, b.hi)}; }
__device__ __forceinline__ Four add(const Four& a, const Four& b) { return {__fadd2_rn(a.lo, b.lo), __fadd2_rn(a.hi, b.hi)}; }
__device__ __forceinline__ Four fma(const Four& a, const Four& b, const Four& c) { return {__ffma2_rn(a.lo, b.lo, c.lo), __ffma2_rn(a.hi, b.hi, c.hi)}; }
__device__ __forceinline__ Four all(float v) { return {make_float2(v, v), make_float2(v, v)}; }
__device__ __forceinline__ float sum(const Four& a) { return (a.lo.x + a.lo.y) + (a.hi.x + a.hi.y); }

// Sum over the warps of a row, in all of them.  `turn` counts the sums, whose places alternate: a warp that is one sum ahead writes
// elsewhere than the others still read.
__device__ __forceinline__ float row_sum(float a, int wide, float (&part)[2][WARPS], int& turn) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) a += __shfl_xor_sync(0xffffffffu, a, d);
  if (wide == 1) return a;
  const int warp = threadIdx.x >> 5, team = warp / wide;
  float(&at)[WARPS] = part[turn & 1];
  ++turn;
  if ((threadIdx.x & 31) == 0) at[warp] = a;
  asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(32 * wide) : "memory");        // (a row's warps alone)
  a = 0.f;
  for (int i = 0; i < wide; ++i) a += at[team * wide + i];
  return a;
}

// -mean / deviation and 1 / deviation of a row (0 and 1 without a norm): v * rstd + shift.  get(j): the j-th four entries; the lane has `mine` of them,
// and zeros behind.
struct Moments {
  float shift, rstd;
};
template <int N, typename Get>
__device__ __forceinline__ Moments moments(const Get& get, int mine, int kind, const ResidualParams& p, float (&part)[2][WARPS], int& turn) {
  if (kind == LQ_NORM_NONE) return {0.f, 1.f};
  Four s = all(0.f);
  if (kind == LQ_NORM_RMS) {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const Four e = get(j);
      s = fma(e, e, s);
    }
    return {0.f, rsqrtf(fmaf(row_sum(sum(s), p.wide, part, turn), p.inv, p.eps))};
  }
#pragma unroll
  for (int j = 0; j < N; ++j) s = add(s, get(j));
  const float mean = row_sum(sum(s), p.wide, part, turn) * p.inv;
  s = all(0.f);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const Four e = add(get(j), all(j < mine ? -mean : 0.f));
    s = fma(e, e, s);
  }
  const float rstd = rsqrtf(fmaf(row_sum(sum(s), p.wide, part, turn), p.inv, p.eps));
  return {-mean * rstd, rstd};
}

template <bool XF32, bool YF32, bool HF32, int N>
__global__ void __launch_bounds__(THREADS) lq_residual_kernel(const __grid_constant__ ResidualParams p) {
  extern __shared__ __align__(16) float4 vectors[];        // [3][features / 4]: factor * gate * weight of N1, weight of N2 * (1 + scale), bias * (1 + scale) + shift
  __shared__ float part[2][WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = WARPS / p.wide, first = (warp % p.wide) * 32 + lane, fours = p.features / 4;
  int turn = 0, held = -1;
  grid_launch_dependents();
  grid_dependency_wait();
  const int step = 32 * p.wide, last = (int)min((long long)p.groups, (blockIdx.x + 1ll) * p.share);
  const int places = first < fours ? (fours - first + step - 1) / step : 0;
  const float4 *va = vectors + first, *vb = va + fours, *vc = vb + fours;
  constexpr int XB = XF32 ? 16 : 8, YB = YF32 ? 16 : 8, HB = HF32 ? 16 : 8;
  for (int g = (int)(blockIdx.x * (long long)p.share); g < last; ++g) {
    const int seq = g / p.seq_groups, in_seq = (g - seq * p.seq_groups) * per + warp / p.wide;
    const long long row = (long long)seq * p.seq_rows + in_seq;
    const int mine = in_seq < p.seq_rows ? places : 0;
    const uint8_t* px = reinterpret_cast<const uint8_t*>(p.x) + row * p.x_row * (XF32 ? 4 : 2) + first * XB;
    const uint8_t* py = reinterpret_cast<const uint8_t*>(p.y) + row * p.y_row * (YF32 ? 4 : 2) + first * YB;
    Raw<XF32> rx[N];
    Raw<YF32> ry[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      rx[j] = Raw<XF32>::zero();
      ry[j] = Raw<YF32>::zero();
      if (j < mine) {
        rx[j] = Raw<XF32>::load(px + j * step * XB);
        if (p.y) ry[j] = Raw<YF32>::load(py + j * step * YB);
      }
    }
    if (seq != held) {                                     // (under the way of the row's loads)
      __syncthreads();
      const long long mod = seq * p.mod_seq;
      for (int i = threadIdx.x; i < fours; i += THREADS) {
        Four a = all(p.factor), b = all(1.f), c = all(0.f), scale = all(0.f);
        if (p.gate) a = mul(a, load4(p.gate, mod + 4 * i, p.mod_f32));
        if (p.after_weight) a = mul(a, load4(p.after_weight, 4 * i, true));
        if (p.weight) b = load4(p.weight, 4 * i, true);
        if (p.bias) c = load4(p.bias, 4 * i, true);
        if (p.scale) scale = load4(p.scale, mod + 4 * i, p.mod_f32);
        b = fma(b, scale, b);
        c = fma(c, scale, c);
        if (p.shift) c = add(c, load4(p.shift, mod + 4 * i, p.mod_f32));
        vectors[i] = make_float4(a.lo.x, a.lo.y, a.hi.x, a.hi.y);
        vectors[fours + i] = make_float4(b.lo.x, b.lo.y, b.hi.x, b.hi.y);
        vectors[2 * fours + i] = make_float4(c.lo.x, c.lo.y, c.hi.x, c.hi.y);
      }
      __syncthreads();
      held = seq;
    }
    const auto open = [](const float4& v) { return Four{make_float2(v.x, v.y), make_float2(v.z, v.w)}; };
    Four x[N];
    if (p.y) {
      const Moments m = moments<N>([&](int j) { return ry[j].open(); }, mine, p.after, p, part, turn);
      const Four rstd = all(m.rstd), off = all(m.shift);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        x[j] = rx[j].open();
        if (j < mine) x[j] = fma(fma(ry[j].open(), rstd, off), open(va[j * step]), x[j]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = rx[j].open();
    }
    if (p.x_out) {
      uint8_t* to = reinterpret_cast<uint8_t*>(p.x_out) + row * p.x_out_row * (XF32 ? 4 : 2) + first * XB;
#pragma unroll
      for (int j = 0; j < N; ++j)
        if (j < mine) Raw<XF32>::store(to + j * step * XB, x[j]);
    }
    if (!p.h) continue;
    const Moments m = moments<N>([&](int j) { return x[j]; }, mine, p.norm, p, part, turn);
    const Four rstd = all(m.rstd), off = all(m.shift);
    uint8_t* to = reinterpret_cast<uint8_t*>(p.h) + row * p.h_row * (HF32 ? 4 : 2) + first * HB;
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (j < mine) Raw<HF32>::store(to + j * step * HB, fma(fma(x[j], rstd, off), open(vb[j * step]), open(vc[j * step])));
  }
}

// fours a lane holds: these, and what lies between takes the next
template <bool XF32, bool YF32, bool HF32, typename F>
cudaError_t with_held(int held, const F& f) {
  return held <= 1   ? f(lq_residual_kernel<XF32, YF32, HF32, 1>)
         : held <= 2 ? f(lq_residual_kernel<XF32, YF32, HF32, 2>)
         : held <= 3 ? f(lq_residual_kernel<XF32, YF32, HF32, 3>)
         : held <= 5 ? f(lq_residual_kernel<XF32, YF32, HF32, 5>)
         : held <= 7 ? f(lq_residual_kernel<XF32, YF32, HF32, 7>)
                     : f(lq_residual_kernel<XF32, YF32, HF32, 9>);
}
template <bool XF32, bool YF32, typename F>
cudaError_t with_h(bool h, int held, const F& f) { return h ? with_held<XF32, YF32, true>(held, f) : with_held<XF32, YF32, false>(held, f); }
template <typename F>
cudaError_t with_types(bool x, bool y, bool h, int held, const F& f) {
  return x ? (y ? with_h<true, true>(h, held, f) : with_h<true, false>(h, held, f)) : (y ? with_h<false, true>(h, held, f) : with_h<false, false>(h, held, f));
}

}  // namespace

extern "C" lq_status lq_residual_norm(const lq_residual* r, void* stream) {
  if (!r || !r->x || (!r->x_out && !r->h) || r->rows < 1 || r->features < 1 || r->sequences < 1) return LQ_ERR_INVALID_ARG;
  if (r->rows % r->sequences != 0) return LQ_ERR_INVALID_ARG;
  for (int32_t n : {r->after, r->norm})
    if (n != LQ_NORM_NONE && n != LQ_NORM_RMS && n != LQ_NORM_LAYER) return LQ_ERR_INVALID_ARG;
  for (int32_t d : {r->x_dtype, r->y_dtype, r->h_dtype, r->mod_dtype})
    if (d != LQ_OUT_F16 && d != LQ_OUT_F32) return LQ_ERR_INVALID_ARG;
  if (!(r->eps >= 0.f) || !isfinite(r->eps) || !isfinite(r->factor)) return LQ_ERR_INVALID_ARG;
  if (!r->y && (r->after != LQ_NORM_NONE || r->gate)) return LQ_ERR_INVALID_ARG;
  if ((r->after_weight && r->after == LQ_NORM_NONE) || (r->weight && r->norm == LQ_NORM_NONE) || (r->bias && r->norm != LQ_NORM_LAYER)) return LQ_ERR_INVALID_ARG;
  if (!r->h && (r->norm != LQ_NORM_NONE || r->scale || r->shift)) return LQ_ERR_INVALID_ARG;
  if (r->features % 8 != 0 || r->features > LQ_MAX_K) return LQ_ERR_UNSUPPORTED;
  const uintptr_t all = (uintptr_t)r->x | (uintptr_t)r->y | (uintptr_t)r->x_out | (uintptr_t)r->h | (uintptr_t)r->after_weight | (uintptr_t)r->weight |
                        (uintptr_t)r->bias | (uintptr_t)r->gate | (uintptr_t)r->scale | (uintptr_t)r->shift;
  if ((all & 15) != 0) return LQ_ERR_INVALID_ARG;
  for (int64_t v : {r->x_row, r->y_row, r->x_out_row, r->h_row, r->mod_seq}) {
    if (v % 8 != 0) return LQ_ERR_INVALID_ARG;
    if (v >= (1ll << 40) || v <= -(1ll << 40)) return LQ_ERR_UNSUPPORTED;
  }
  // Where outputs may lie: on no input but, entry on entry, x' on x and h on y.
  const auto rows = [&](const void* at, int64_t step, int32_t dt) {
    const int64_t esz = dt == LQ_OUT_F32 ? 4 : 2;
    return LqRuns{(uintptr_t)at, {step * esz, 0, 0}, {r->rows, 1, 1}, r->features * esz};
  };
  const auto line = [&](const void* at, int64_t step, int64_t n, int64_t esz) {
    return LqRuns{(uintptr_t)at, {step * esz, 0, 0}, {n, 1, 1}, r->features * esz};
  };
  const auto status = [](LqPlaces c) { return c == LQ_APART ? LQ_OK : c == LQ_SHARED ? LQ_ERR_INVALID_ARG : LQ_ERR_UNSUPPORTED; };
  const bool x_in_place = r->x_out == r->x && r->x_out_row == r->x_row;
  const bool h_in_place = r->h && r->h == r->y && r->h_row == r->y_row && r->h_dtype == r->y_dtype;
  LqRuns out[2], in[8];
  int n_in = 0;
  if (r->y) in[n_in++] = rows(r->y, r->y_row, r->y_dtype);
  in[n_in++] = rows(r->x, r->x_row, r->x_dtype);
  for (const float* w : {r->after_weight, r->weight, r->bias})
    if (w) in[n_in++] = line(w, 0, 1, 4);
  for (const void* m : {r->gate, r->scale, r->shift})
    if (m) in[n_in++] = line(m, r->sequences == 1 ? 0 : r->mod_seq, r->sequences, r->mod_dtype == LQ_OUT_F32 ? 4 : 2);
  const int at_x = r->y ? 1 : 0;
  int n_out = 0;
  lq_status s = LQ_OK;
  if (r->x_out) out[n_out++] = rows(r->x_out, r->x_out_row, r->x_dtype);
  if (r->h) out[n_out++] = rows(r->h, r->h_row, r->h_dtype);
  for (int i = 0; i < n_out && s == LQ_OK; ++i) {
    const bool is_h = r->h && i == n_out - 1;
    s = status(lq_runs_collide(out[i]));
    for (int j = 0; j < n_in && s == LQ_OK; ++j) {
      if (!is_h && j == at_x && x_in_place) continue;
      if (is_h && r->y && j == 0 && h_in_place) continue;
      s = status(lq_runs_meet(out[i], in[j]));
    }
  }
  if (s == LQ_OK && n_out == 2) s = status(lq_runs_meet(out[0], out[1]));
  if (s != LQ_OK) return s;
  const int sms = lq_device_sms(r->device);
  if (sms == 0) return LQ_ERR_CUDA;
  LqDeviceGuard guard(r->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  ResidualParams p = {};
  p.x = r->x; p.y = r->y; p.x_out = r->x_out; p.h = r->h;
  p.x_row = r->x_row; p.y_row = r->y_row; p.x_out_row = r->x_out_row; p.h_row = r->h_row;
  p.after_weight = r->after_weight; p.weight = r->weight; p.bias = r->bias;
  p.gate = r->gate; p.scale = r->scale; p.shift = r->shift;
  const bool one = !(r->gate || r->scale || r->shift) || r->mod_seq == 0 || r->sequences == 1;
  p.mod_seq = one ? 0 : r->mod_seq;
  p.rows = r->rows; p.features = r->features; p.seq_rows = one ? r->rows : r->rows / r->sequences;
  p.after = r->after; p.norm = r->norm; p.mod_f32 = r->mod_dtype == LQ_OUT_F32;
  p.factor = r->factor; p.eps = r->eps; p.inv = 1.f / (float)r->features;
  // The fewest warps that hold a row; more of them where a sequence has fewer rows than a thread block would take, and with rows too few to give
  // every SM eight warps, for then a row's own time is what counts.
  const int fours = r->features / 4;
  p.wide = 1;
  while (32 * p.wide * 9 < fours || (p.wide < WARPS && 32 * p.wide < fours && (p.seq_rows * p.wide < WARPS || (long long)r->rows * p.wide < 8ll * sms)))
    p.wide *= 2;
  const int per = WARPS / p.wide, held = lq_ceil_div(fours, 32 * p.wide);
  p.seq_groups = 1 + (p.seq_rows - 1) / per;
  p.groups = p.seq_groups * (p.rows / p.seq_rows);
  const size_t smem = 3 * (size_t)p.features * sizeof(float);
  const auto launch = [&](auto* kernel) {
    // (the widest call's: the limit is the kernel's, for all threads, and a call that set its own would lower it under another's launch)
    const int most = 3 * LQ_MAX_K * (int)sizeof(float);
    const cudaError_t c = smem > 47 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) : cudaSuccess;
    if (c != cudaSuccess) return c;
    // Neighbouring groups to a thread block, as many blocks as are resident at once: with seven and nine fours a lane two an SM (us of 32768 rows of
    // 2240, fp32 stream, with 2 / 3 / 4 / 8 / 16 blocks an SM: 151 / 184 / 153 / 158 / 175; of 8192 rows of 1152 14.9 / 19.5 / 16.7 / 19.7 / 19.6; with 2 / 3 /
    // 4 / 8: 16384 rows of 4096, fp32 stream 147 / 182 / 151 / 159, fp16 117 / 145 / 122 / 128; 8192 of 8192, fp32 171 / 207 / 178 / 189, fp16 137 / 166 / 145 /
    // 153; 20000 of 3200, fp16 121 / 149 / 125 / 133).  Of the other numbers one has been timed, five fours a lane (20000 rows of 5120, fp16: 237 / 179 /
    // 223 / 197): three would be better there than the four that it takes.
    p.share = 1 + (p.groups - 1) / (sms * (held > 5 ? 2 : held > 2 ? 4 : 8));
    return lq_launch(kernel, 1 + (p.groups - 1) / p.share, THREADS, smem, (cudaStream_t)stream, p);
  };
  const cudaError_t e = with_types(r->x_dtype == LQ_OUT_F32, r->y && r->y_dtype == LQ_OUT_F32, r->h_dtype == LQ_OUT_F32, held, launch);
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
