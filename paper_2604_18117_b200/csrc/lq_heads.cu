// Queries and keys behind a projection: norm of each head and rotation of its leading entries by the row's position, in one pass.
//
//   z = x / sqrt(mean x^2 + eps) * w          or   (x - mean) / sqrt(var + eps) * w + b          (head of D entries)
//   (u, v) -> (u cos t - v sin t, v cos t + u sin t),   t = pos[axis of the pair] * frequency of the pair
//
// Angles.  A frequency is kept as a 64-bit fraction of a turn, F = 2^64 frac(f / 2 pi); pos * F modulo 2^64 is the exact fraction of a
// turn that the rounded F gives at an int32 position, so that an angle is off by 2^31 * 2^-65 turns (4e-10 radians) at most.  The nearest
// quarter turn is taken off in integers and only the rest, at most an eighth of a turn, becomes a float.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>
#include <new>
#include <vector>

#include "lq_device.cuh"
#include "lq_internal.h"

using namespace lqdev;

struct lq_rope {
  int axes, pairs, halves, device;
  uint64_t* d_turn;   // [pairs] fraction of a turn a position, 2^64 = 1
  uint8_t* d_axis;    // [pairs]
};

namespace {

constexpr int MAX_D = 256, WARPS = 8;
enum { ROT_NONE = 0, ROT_PAIRS = 1, ROT_HALVES = 2 };

struct Side {
  const void* in;
  void* out;
  long long in_seq, in_row, in_head, out_seq, out_row, out_head;
  const float *weight, *bias;
};
struct HeadsParams {
  Side side[2];
  int tasks;                    // rows * parts: a warp's work is a row's heads of one part
  int heads, q_heads, parts, part_heads, seq_len, lanes, groups, axes, pairs;
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
__device__ __forceinline__ void open8(const Raw<__half>& r, float (&x)[8]) {
  const uint32_t w[4] = {r.a.x, r.a.y, r.b.x, r.b.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void open8(const Raw<float>& r, float (&x)[8]) {
  x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w; x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
template <bool SPLIT>
__device__ __forceinline__ void store8(__half* p, int apart, const float (&x)[8]) {
  uint4 v;
  __half2* h = reinterpret_cast<__half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
  if constexpr (SPLIT) {
    *reinterpret_cast<uint2*>(p) = make_uint2(v.x, v.y);
    *reinterpret_cast<uint2*>(p + apart) = make_uint2(v.z, v.w);
  } else {
    *reinterpret_cast<uint4*>(p) = v;
  }
}
template <bool SPLIT>
__device__ __forceinline__ void store8(float* p, int apart, const float (&x)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
  *reinterpret_cast<float4*>(p + (SPLIT ? apart : 4)) = make_float4(x[4], x[5], x[6], x[7]);
}

__device__ __forceinline__ float2 cos_sin(uint64_t turn, int32_t pos) {
  const int32_t t = (int32_t)(uint32_t)((turn * (uint64_t)(int64_t)pos) >> 32);       // fraction of a turn, 2^32 = 1
  const int32_t quarter = (int32_t)(((uint32_t)t + 0x20000000u) >> 30);                // nearest quarter turn, 0 .. 3
  const int32_t rest = (int32_t)((uint32_t)t - ((uint32_t)quarter << 30));             // [-2^29, 2^29)
  float s, c;
  sincospif((float)rest * 0x1p-31f, &s, &c);
  float2 r = (quarter & 1) ? make_float2(-s, c) : make_float2(c, s);
  if (quarter & 2) r = make_float2(-r.x, -r.y);
  return r;
}

// Sum over the `lanes` neighbours of a group, in every lane of it.  lanes is a power of two (then xor steps do) or not.
__device__ __forceinline__ float group_sum(float a, int lanes, int at, int lane) {
  if ((lanes & (lanes - 1)) == 0) {
    for (int d = lanes >> 1; d > 0; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
    return a;
  }
  for (int d = 1; d < lanes; d *= 2) {
    const float u = __shfl_down_sync(0xffffffffu, a, d);
    if (at + d < lanes) a += u;
  }
  return __shfl_sync(0xffffffffu, a, lane - at);
}

// A warp takes a row and walks over its heads (or over a part of them, where rows are few): D / 8 lanes hold a head, 32 / (D / 8) heads are in
// hand at once.  A lane's eight entries are the two sides of the same four pairs in every head, so the row's angles are formed once, in the lane
// that needs them, and nothing passes through shared memory; the norm's sum crosses the head's lanes by shuffles.
template <typename TIN, typename TOUT, int NORM, int ROT>
__global__ void __launch_bounds__(32 * WARPS) lq_heads_kernel(const __grid_constant__ HeadsParams p) {
  constexpr bool SPLIT = ROT == ROT_HALVES;
  constexpr int U = sizeof(TIN) == 4 ? 2 : 4;             // heads of a lane whose loads are in flight together
  const int lane = threadIdx.x & 31, V = p.lanes;
  const int task = blockIdx.x * WARPS + (threadIdx.x >> 5);
  const int grp = lane / V, v = lane - grp * V;
  const bool works = grp < p.groups;
  // pairs 4 v .. 4 v + 3: entries 8 v .. 8 v + 7, or (halves) 4 v .. 4 v + 3 and as many half of the rotated part further; what is not rotated lies
  // behind, eight neighbours a lane
  const bool turned = ROT != ROT_NONE && 4 * v < p.pairs;
  const int first = SPLIT && turned ? 4 * v : 8 * v, apart = SPLIT && turned ? p.pairs : 4;
  uint64_t turn[4];
  int axis[4];
  if constexpr (ROT != ROT_NONE) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int i = min(4 * v + j, p.pairs - 1);
      turn[j] = p.turn[i];
      axis[j] = p.axis[i];
    }
  }
  grid_launch_dependents();
  grid_dependency_wait();
  if (task >= p.tasks) return;
  const int row = task / p.parts, part = task - row * p.parts;
  const int seq = row / p.seq_len, at = row - seq * p.seq_len;
  const int h_begin = part * p.part_heads, h_end = min(p.heads, h_begin + p.part_heads);
  float2 cs[4];
  bool have_angles = false;
  for (int side = 0; side < 2; ++side) {
    const Side& s = p.side[side];
    const int begin = max(h_begin - (side ? p.q_heads : 0), 0), end = min(h_end, side ? p.heads : p.q_heads) - (side ? p.q_heads : 0);
    if (begin >= end) continue;
    const TIN* in = reinterpret_cast<const TIN*>(s.in) + seq * s.in_seq + at * s.in_row + first;
    TOUT* out = reinterpret_cast<TOUT*>(s.out) + seq * s.out_seq + at * s.out_row + first;
    float w[8], b[8];
    if constexpr (NORM != LQ_NORM_NONE) {
#pragma unroll
      for (int j = 0; j < 8; ++j) { w[j] = 1.f; b[j] = 0.f; }
      if (works && s.weight) open8(load_raw<SPLIT>(s.weight + first, apart), w);
      if (NORM == LQ_NORM_LAYER && works && s.bias) open8(load_raw<SPLIT>(s.bias + first, apart), b);
    }
    for (int h0 = begin; h0 < end; h0 += U * p.groups) {
      Raw<TIN> raw[U] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * p.groups + grp;
        if (works && h < end) raw[u] = load_raw<SPLIT>(in + h * s.in_head, apart);
      }
      if constexpr (ROT != ROT_NONE) {
        if (!have_angles) {                               // under the first loads
#pragma unroll
          for (int j = 0; j < 4; ++j) cs[j] = cos_sin(turn[j], p.pos[(long long)row * p.axes + axis[j]]);
          have_angles = true;
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (h0 + u * p.groups >= end) break;              // (the whole warp)
        const int h = h0 + u * p.groups + grp;
        float x[8];
        open8(raw[u], x);
        if constexpr (NORM != LQ_NORM_NONE) {
          float m = 0.f, a = 0.f;
          if constexpr (NORM == LQ_NORM_LAYER) {
#pragma unroll
            for (int j = 0; j < 8; ++j) m += x[j];
            m = group_sum(m, V, v, lane) * p.inv_d;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            x[j] -= m;
            a = fmaf(x[j], x[j], a);
          }
          a = group_sum(a, V, v, lane);
          const float rstd = rsqrtf(fmaf(a, p.inv_d, p.eps));
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = NORM == LQ_NORM_LAYER ? fmaf(x[j] * rstd, w[j], b[j]) : x[j] * rstd * w[j];
        }
        if (ROT != ROT_NONE && turned) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int lo = SPLIT ? j : 2 * j, hi = SPLIT ? j + 4 : 2 * j + 1;
            const float a = x[lo], c = x[hi];
            if (SPLIT || 4 * v + j < p.pairs) {           // (halves turn whole lanes)
              x[lo] = a * cs[j].x - c * cs[j].y;
              x[hi] = c * cs[j].x + a * cs[j].y;
            }
          }
        }
        if (works && h < end) store8<SPLIT>(out + h * s.out_head, apart, x);
      }
    }
  }
}

template <typename TIN, typename TOUT, int NORM, int ROT>
cudaError_t launch(const HeadsParams& p, cudaStream_t st) {
  return lq_launch(lq_heads_kernel<TIN, TOUT, NORM, ROT>, (p.tasks + WARPS - 1) / WARPS, 32 * WARPS, 0, st, p);
}
template <typename TIN, typename TOUT, int NORM>
cudaError_t launch_rot(const HeadsParams& p, int rot, cudaStream_t st) {
  return rot == ROT_NONE ? launch<TIN, TOUT, NORM, ROT_NONE>(p, st) : rot == ROT_PAIRS ? launch<TIN, TOUT, NORM, ROT_PAIRS>(p, st) : launch<TIN, TOUT, NORM, ROT_HALVES>(p, st);
}
template <typename TIN, typename TOUT>
cudaError_t launch_norm(const HeadsParams& p, int norm, int rot, cudaStream_t st) {
  return norm == LQ_NORM_NONE ? launch_rot<TIN, TOUT, LQ_NORM_NONE>(p, rot, st)
         : norm == LQ_NORM_RMS ? launch_rot<TIN, TOUT, LQ_NORM_RMS>(p, rot, st) : launch_rot<TIN, TOUT, LQ_NORM_LAYER>(p, rot, st);
}

// Strides over dimensions of one entry mean nothing; the others keep entries on 16-byte boundaries, and no two outputs on one place.
lq_status take_side(const lq_heads* h, int sequences, int seq_len, lq_norm norm, Side* s) {
  if (!h->in || !h->out || h->heads < 1) return LQ_ERR_INVALID_ARG;
  if (h->heads > 4096) return LQ_ERR_UNSUPPORTED;
  if ((((uintptr_t)h->in | (uintptr_t)h->out | (uintptr_t)h->weight | (uintptr_t)h->bias) & 15) != 0) return LQ_ERR_INVALID_ARG;
  if ((h->weight && norm == LQ_NORM_NONE) || (h->bias && norm != LQ_NORM_LAYER)) return LQ_ERR_INVALID_ARG;
  *s = Side{h->in, h->out, h->in_seq, h->in_row, h->in_head, h->out_seq, h->out_row, h->out_head, h->weight, h->bias};
  if (sequences == 1) s->in_seq = s->out_seq = 0;
  if (seq_len == 1) s->in_row = s->out_row = 0;
  if (h->heads == 1) s->in_head = s->out_head = 0;
  for (long long v : {s->in_seq, s->in_row, s->in_head, s->out_seq, s->out_row, s->out_head})
    if (v % 8 != 0) return LQ_ERR_INVALID_ARG;
  if ((sequences > 1 && s->out_seq == 0) || (seq_len > 1 && s->out_row == 0) || (h->heads > 1 && s->out_head == 0)) return LQ_ERR_INVALID_ARG;
  return LQ_OK;
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
        if (freq && !isfinite(freq[i])) return LQ_ERR_NUMERIC;
        const long double f = freq ? (long double)freq[i]
                                   : powl((long double)cfg->theta, -2.0L * (cfg->shared ? i : j) / (cfg->shared ? rot : cfg->dims[a]));
        long double t = f / (2.0L * acosl(-1.0L));
        if (!isfinite(t)) return LQ_ERR_NUMERIC;
        t -= floorl(t);                                      // [0, 1]: 1 itself wraps to 0 below
        const long double scaled = roundl(ldexpl(t, 64));
        turn.push_back(scaled >= 0x1p64L ? 0 : (uint64_t)scaled);
        which.push_back((uint8_t)(axis ? axis[i] : a));
      }
  } catch (const std::bad_alloc&) { return LQ_ERR_ALLOC; }
  int ndev = 0;
  if (lq_note_cuda(cudaGetDeviceCount(&ndev)) != cudaSuccess || device < 0 || device >= ndev) return LQ_ERR_CUDA;
  LqDeviceGuard guard(device);
  if (!guard.ok) return LQ_ERR_CUDA;
  lq_rope* R = new (std::nothrow) lq_rope{cfg->axes, rot / 2, cfg->halves, device, nullptr, nullptr};
  if (!R) return LQ_ERR_ALLOC;
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

extern "C" lq_status lq_qk_norm_rope(const lq_heads* q, const lq_heads* k, int32_t head_dim, int32_t sequences, int32_t seq_len, lq_norm norm,
                                     float eps, const lq_rope* R, const int32_t* pos, lq_out_dtype in_dtype, lq_out_dtype out_dtype, void* stream) {
  if (!R || (!q && !k) || sequences < 1 || seq_len < 1 || head_dim < 1) return LQ_ERR_INVALID_ARG;
  if (norm != LQ_NORM_NONE && norm != LQ_NORM_RMS && norm != LQ_NORM_LAYER) return LQ_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !isfinite(eps)) return LQ_ERR_INVALID_ARG;
  for (lq_out_dtype d : {in_dtype, out_dtype})
    if (d != LQ_OUT_F16 && d != LQ_OUT_F32) return LQ_ERR_INVALID_ARG;
  if (head_dim % 8 != 0 || head_dim > MAX_D) return LQ_ERR_UNSUPPORTED;
  if (2 * R->pairs > head_dim || (R->pairs > 0 && !pos) || ((uintptr_t)pos & 3) != 0) return LQ_ERR_INVALID_ARG;
  const long long rows = (long long)sequences * seq_len;
  if (rows > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  HeadsParams p = {};
  lq_status s;
  if (q && (s = take_side(q, sequences, seq_len, norm, &p.side[0])) != LQ_OK) return s;
  if (k && (s = take_side(k, sequences, seq_len, norm, &p.side[1])) != LQ_OK) return s;
  p.q_heads = q ? q->heads : 0;
  p.heads = p.q_heads + (k ? k->heads : 0);
  p.lanes = head_dim / 8;
  p.groups = 32 / p.lanes;
  // A warp walks over all heads of its row once there are warps enough to fill the GPU; below that the heads are spread over more warps.
  const long long walk = lq_ceil_div(p.heads, p.groups), fill = 148 * 32;
  const long long parts = std::max(1ll, std::min(walk, fill / rows));
  p.part_heads = (int)((walk + parts - 1) / parts) * p.groups;
  p.parts = lq_ceil_div(p.heads, p.part_heads);
  if (rows * p.parts > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  p.tasks = (int)(rows * p.parts);
  p.seq_len = seq_len; p.axes = R->axes; p.pairs = R->pairs;
  p.eps = eps; p.inv_d = 1.f / (float)head_dim;
  p.turn = R->d_turn; p.axis = R->d_axis; p.pos = pos;
  LqDeviceGuard guard(R->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  const int rot = R->pairs == 0 ? ROT_NONE : R->halves ? ROT_HALVES : ROT_PAIRS;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e =
      in_dtype == LQ_OUT_F16 ? (out_dtype == LQ_OUT_F16 ? launch_norm<__half, __half>(p, norm, rot, st) : launch_norm<__half, float>(p, norm, rot, st))
                             : (out_dtype == LQ_OUT_F16 ? launch_norm<float, __half>(p, norm, rot, st) : launch_norm<float, float>(p, norm, rot, st));
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
