// The residual stream between two blocks, in one pass over its rows:
//
//   x' = x + factor * gate * N1(y),   h = (N2(x') * w + b) * (1 + scale) + shift
//
// N: none, RMS or LayerNorm of a row; gate, scale and shift are a sequence's.  Reads x and y once and writes x' and h once; the memory
// bounds it.  A row is held in registers by one, two or four warps, up to nine times eight neighbouring entries a lane, all asked for at once and
// kept as they lie in memory until they are used: with few warps of many loads each no row waits for another's, and most sums stay within
// a warp.  Variances are sums about the mean that is known; h is made of x' before that is rounded to its type.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "lq_device.cuh"
#include "lq_heads_places.h"
#include "lq_internal.h"

using namespace lqdev;

namespace {

constexpr int THREADS = 128, WARPS = THREADS / 32;

struct ResidualParams {
  const void *x, *y;
  void *x_out, *h;
  long long x_row, y_row, x_out_row, h_row, mod_seq;
  const float *after_weight, *weight, *bias;
  const void *gate, *scale, *shift;
  int rows, features, seq_rows, after, norm, h_f32, mod_f32, wide;     // wide: warps of a row
  float factor, eps, inv;
};

struct Eight {
  float v[8];
};
template <bool F32> struct Raw;
template <> struct Raw<false> {
  uint4 a;
  __device__ __forceinline__ static Raw load(const void* p, long long at) { return {*reinterpret_cast<const uint4*>(reinterpret_cast<const __half*>(p) + at)}; }
  __device__ __forceinline__ static Raw zero() { return {make_uint4(0, 0, 0, 0)}; }
  __device__ __forceinline__ Eight open() const {
    Eight e;
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
      e.v[2 * i] = f.x; e.v[2 * i + 1] = f.y;
    }
    return e;
  }
};
template <> struct Raw<true> {
  float4 a, b;
  __device__ __forceinline__ static Raw load(const void* p, long long at) {
    const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + at);
    return {q[0], q[1]};
  }
  __device__ __forceinline__ static Raw zero() { return {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}; }
  __device__ __forceinline__ Eight open() const { return {{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w}}; }
};
__device__ __forceinline__ Eight load8(const void* p, long long at, bool f32) { return f32 ? Raw<true>::load(p, at).open() : Raw<false>::load(p, at).open(); }
__device__ __forceinline__ void store8(void* p, long long at, bool f32, const Eight& e) {
  if (f32) {
    float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + at);
    q[0] = make_float4(e.v[0], e.v[1], e.v[2], e.v[3]);
    q[1] = make_float4(e.v[4], e.v[5], e.v[6], e.v[7]);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(e.v[2 * i], e.v[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(reinterpret_cast<__half*>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// Sum over the warps of a row, in all of them.  `turn` counts the sums, whose places alternate: a warp that is one sum ahead writes
// elsewhere than the others still read.
__device__ __forceinline__ float row_sum(float a, int wide, float (&part)[2][WARPS], int& turn) {
#pragma unroll
  for (int d = 16; d > 0; d /= 2) a += __shfl_xor_sync(0xffffffffu, a, d);
  if (wide == 1) return a;
  const int warp = threadIdx.x >> 5;
  float(&at)[WARPS] = part[turn & 1];
  ++turn;
  if ((threadIdx.x & 31) == 0) at[warp] = a;
  __syncthreads();
  const int first = warp / wide * wide;
  a = 0.f;
  for (int i = 0; i < wide; ++i) a += at[first + i];
  return a;
}

// Mean and 1 / deviation of a row (0 and 1 without a norm): (v - mean) * rstd.  get(j): the j-th eight entries, zeros where the lane has none.
struct Moments {
  float mean, rstd;
};
template <int N, typename Get>
__device__ __forceinline__ Moments moments(const Get& get, const bool (&live)[N], int kind, const ResidualParams& p, float (&part)[2][WARPS], int& turn) {
  Moments m{0.f, 1.f};
  if (kind == LQ_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const Eight e = get(j);
#pragma unroll
      for (int i = 0; i < 8; ++i) s += e.v[i];
    }
    m.mean = row_sum(s, p.wide, part, turn) * p.inv;
  }
  if (kind != LQ_NORM_NONE) {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const Eight e = get(j);
      const float off = live[j] ? m.mean : 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) s = fmaf(e.v[i] - off, e.v[i] - off, s);
    }
    m.rstd = rsqrtf(fmaf(row_sum(s, p.wide, part, turn), p.inv, p.eps));
  }
  return m;
}

template <bool XF32, bool YF32, int N>
__global__ void __launch_bounds__(THREADS) lq_residual_kernel(const __grid_constant__ ResidualParams p) {
  __shared__ float part[2][WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = WARPS / p.wide, first = (warp % p.wide) * 32 + lane;
  int turn = 0;
  grid_launch_dependents();
  grid_dependency_wait();
  const int groups = (p.rows + per - 1) / per;
  for (int g = blockIdx.x; g < groups; g += gridDim.x) {
    const long long row = (long long)g * per + warp / p.wide;
    const bool real = row < p.rows;
    bool live[N];
    Raw<XF32> rx[N];
    Raw<YF32> ry[N];
    const auto at = [&](int j) { return 8 * (first + 32 * p.wide * j); };
#pragma unroll
    for (int j = 0; j < N; ++j) {
      live[j] = real && at(j) < p.features;
      rx[j] = Raw<XF32>::zero();
      ry[j] = Raw<YF32>::zero();
      if (live[j]) {
        rx[j] = Raw<XF32>::load(p.x, row * p.x_row + at(j));
        if (p.y) ry[j] = Raw<YF32>::load(p.y, row * p.y_row + at(j));
      }
    }
    const long long mod = real ? row / p.seq_rows * p.mod_seq : 0;
    Eight x[N];
    const Moments my = p.y ? moments<N>([&](int j) { return ry[j].open(); }, live, p.after, p, part, turn) : Moments{0.f, 1.f};
#pragma unroll
    for (int j = 0; j < N; ++j) {
      x[j] = rx[j].open();
      if (!live[j]) continue;
      if (p.y) {
        Eight y = ry[j].open();
#pragma unroll
        for (int i = 0; i < 8; ++i) y.v[i] = (y.v[i] - my.mean) * my.rstd;
        if (p.after_weight) {
          const Eight w = load8(p.after_weight, at(j), true);
#pragma unroll
          for (int i = 0; i < 8; ++i) y.v[i] *= w.v[i];
        }
        if (p.gate) {
          const Eight w = load8(p.gate, mod + at(j), p.mod_f32);
#pragma unroll
          for (int i = 0; i < 8; ++i) y.v[i] *= w.v[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j].v[i] = fmaf(p.factor, y.v[i], x[j].v[i]);
      }
      if (p.x_out) store8(p.x_out, row * p.x_out_row + at(j), XF32, x[j]);
    }
    if (!p.h) continue;
    const Moments mx = moments<N>([&](int j) { return x[j]; }, live, p.norm, p, part, turn);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      if (!live[j]) continue;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[j].v[i] = (x[j].v[i] - mx.mean) * mx.rstd;
      if (p.weight) {
        const Eight w = load8(p.weight, at(j), true);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j].v[i] *= w.v[i];
      }
      if (p.bias) {
        const Eight w = load8(p.bias, at(j), true);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j].v[i] += w.v[i];
      }
      if (p.scale) {
        const Eight w = load8(p.scale, mod + at(j), p.mod_f32);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j].v[i] = fmaf(x[j].v[i], w.v[i], x[j].v[i]);
      }
      if (p.shift) {
        const Eight w = load8(p.shift, mod + at(j), p.mod_f32);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[j].v[i] += w.v[i];
      }
      store8(p.h, row * p.h_row + at(j), p.h_f32, x[j]);
    }
  }
}

// eights a lane holds: these, and what lies between takes the next
template <bool XF32, bool YF32>
cudaError_t launch_held(const ResidualParams& p, int held, int blocks, cudaStream_t st) {
  const auto launch = [&](auto* kernel) { return lq_launch(kernel, blocks, THREADS, 0, st, p); };
  return held == 1   ? launch(lq_residual_kernel<XF32, YF32, 1>)
         : held == 2 ? launch(lq_residual_kernel<XF32, YF32, 2>)
         : held == 3 ? launch(lq_residual_kernel<XF32, YF32, 3>)
         : held <= 5 ? launch(lq_residual_kernel<XF32, YF32, 5>)
         : held <= 7 ? launch(lq_residual_kernel<XF32, YF32, 7>)
                     : launch(lq_residual_kernel<XF32, YF32, 9>);
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
  ResidualParams p = {r->x, r->y, r->x_out, r->h, r->x_row, r->y_row, r->x_out_row, r->h_row, r->sequences == 1 ? 0 : r->mod_seq, r->after_weight, r->weight,
                      r->bias, r->gate, r->scale, r->shift, r->rows, r->features, r->rows / r->sequences, r->after, r->norm,
                      r->h_dtype == LQ_OUT_F32, r->mod_dtype == LQ_OUT_F32, 1, r->factor, r->eps, 1.f / (float)r->features};
  int ndev = 0;
  if (lq_note_cuda(cudaGetDeviceCount(&ndev)) != cudaSuccess || r->device < 0 || r->device >= ndev) return LQ_ERR_CUDA;
  LqDeviceGuard guard(r->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  int sms = 0;
  if (lq_note_cuda(cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, r->device)) != cudaSuccess) return LQ_ERR_CUDA;
  // The fewest warps that hold a row; with rows too few to give every SM eight warps more of them, for then a row's own time is what counts.
  const int chunks = r->features / 8;
  while (32 * p.wide * 9 < chunks || (p.wide < WARPS && 32 * p.wide < chunks && (long long)r->rows * p.wide < 8ll * sms)) p.wide *= 2;
  const int held = lq_ceil_div(chunks, 32 * p.wide), groups = lq_ceil_div(r->rows, WARPS / p.wide), blocks = std::min(groups, sms * 32);
  const bool xf = r->x_dtype == LQ_OUT_F32, yf = r->y && r->y_dtype == LQ_OUT_F32;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e = xf ? (yf ? launch_held<true, true>(p, held, blocks, st) : launch_held<true, false>(p, held, blocks, st))
                           : (yf ? launch_held<false, true>(p, held, blocks, st) : launch_held<false, false>(p, held, blocks, st));
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
