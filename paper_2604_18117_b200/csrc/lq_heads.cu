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

constexpr int MAX_D = 256, NTHREADS = 256, ITER = 2;
enum { ROT_NONE = 0, ROT_PAIRS = 1, ROT_HALVES = 2 };

struct Side {
  const void* in;
  void* out;
  long long in_seq, in_row, in_head, out_seq, out_row, out_head;
  const float *weight, *bias;
};
struct HeadsParams {
  Side side[2];
  long long items;              // rows * heads
  int heads, q_heads, seq_len, axes, pairs;
  float eps, inv_d;
  const uint64_t* turn;
  const uint8_t* axis;
  const int32_t* pos;
};

// eight neighbouring entries
__device__ __forceinline__ void load8(const __half* p, float (&x)[8]) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  const __half2* h = reinterpret_cast<const __half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(h[i]);
    x[2 * i] = f.x; x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}
__device__ __forceinline__ void store8(__half* p, const float (&x)[8]) {
  uint4 v;
  __half2* h = reinterpret_cast<__half2*>(&v);
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
  *reinterpret_cast<uint4*>(p) = v;
}
__device__ __forceinline__ void store8(float* p, const float (&x)[8]) {
  reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
  reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
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

// Block: V = D / 8 threads to a head, as many heads as fit 256 threads, ITER of those one behind the other.  Heads of a row are
// neighbours, so a block sees few rows and forms their angles once.
template <typename TIN, typename TOUT, int NORM, int ROT>
__global__ void __launch_bounds__(NTHREADS) lq_heads_kernel(const __grid_constant__ HeadsParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int V = blockDim.x, HB = blockDim.y, v = threadIdx.x, y = threadIdx.y, tid = y * V + v;
  float2* red = reinterpret_cast<float2*>(smem);                          // [HB][V]
  float* xbuf = reinterpret_cast<float*>(red + ((HB * V + 1) & ~1));      // [HB][8 V] (ROT_HALVES), on 16 bytes
  float2* trig = reinterpret_cast<float2*>(xbuf + (ROT == ROT_HALVES ? HB * V * 8 : 0));   // [rows][pairs]
  const long long item0 = (long long)blockIdx.x * (HB * ITER);
  const long long items = min((long long)(HB * ITER), p.items - item0);
  const long long row0 = item0 / p.heads;
  grid_launch_dependents();
  grid_dependency_wait();

  float x[ITER][8];
  const Side* side[ITER];
  long long out[ITER];
  int row_at[ITER];
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const long long at = (long long)i * HB + y;
    if (at < items) {
      const long long item = item0 + at, row = item / p.heads;
      const int head = (int)(item - row * p.heads);
      const bool is_k = head >= p.q_heads;
      const Side& s = p.side[is_k];
      const int h = is_k ? head - p.q_heads : head;
      const long long b = row / p.seq_len, r = row - b * p.seq_len;
      side[i] = &s;
      row_at[i] = (int)(row - row0);
      load8(reinterpret_cast<const TIN*>(s.in) + b * s.in_seq + r * s.in_row + h * s.in_head + 8 * v, x[i]);
      out[i] = b * s.out_seq + r * s.out_row + h * s.out_head + 8 * v;
    }
  }
  if constexpr (ROT != ROT_NONE) {
    const int rows = (int)((item0 + items - 1) / p.heads - row0) + 1;
    for (int e = tid; e < rows * p.pairs; e += HB * V) {
      const int r = e / p.pairs, j = e - r * p.pairs;
      trig[e] = cos_sin(p.turn[j], p.pos[(row0 + r) * p.axes + p.axis[j]]);
    }
    if constexpr (NORM == LQ_NORM_NONE) __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < ITER; ++i) {
    const bool live = (long long)i * HB + y < items;
    if constexpr (NORM != LQ_NORM_NONE) {
      if (live) {
        float a = 0.f, m = 0.f;
        if constexpr (NORM == LQ_NORM_LAYER) {
#pragma unroll
          for (int j = 0; j < 8; ++j) m += x[i][j];
          m *= 0.125f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) a = fmaf(x[i][j] - m, x[i][j] - m, a);
        red[tid] = make_float2(a, m);
      }
      __syncthreads();
      if (live) {
        float a = 0.f, m = 0.f;
        for (int j = 0; j < V; ++j) { a += red[y * V + j].x; m += red[y * V + j].y; }
        if constexpr (NORM == LQ_NORM_LAYER) {
          m *= 8.f * p.inv_d;
          float d = 0.f;
          for (int j = 0; j < V; ++j) d = fmaf(red[y * V + j].y - m, red[y * V + j].y - m, d);
          a = fmaf(8.f, d, a);
        }
        const float rstd = 1.f / sqrtf(fmaf(a, p.inv_d, p.eps));
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] = (x[i][j] - m) * rstd;
        if (side[i]->weight) {
          float w[8];
          load8(side[i]->weight + 8 * v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[i][j] *= w[j];
        }
        if (NORM == LQ_NORM_LAYER && side[i]->bias) {
          float w[8];
          load8(side[i]->bias + 8 * v, w);
#pragma unroll
          for (int j = 0; j < 8; ++j) x[i][j] += w[j];
        }
      }
    }
    if constexpr (ROT == ROT_HALVES) {
      if (live) {
        float4* b = reinterpret_cast<float4*>(xbuf + 8 * tid);
        b[0] = make_float4(x[i][0], x[i][1], x[i][2], x[i][3]);
        b[1] = make_float4(x[i][4], x[i][5], x[i][6], x[i][7]);
      }
    }
    __syncthreads();      // the partners' entries are there; the sums of this heads' group have been read
    if (live) {
      if constexpr (ROT == ROT_PAIRS) {
        const float2* cs = trig + row_at[i] * p.pairs + 4 * v;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * v + j < p.pairs) {
            const float2 t = cs[j];
            const float u = x[i][2 * j], w = x[i][2 * j + 1];
            x[i][2 * j] = u * t.x - w * t.y;
            x[i][2 * j + 1] = w * t.x + u * t.y;
          }
      }
      if constexpr (ROT == ROT_HALVES) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {                     // half of the rotated part is a multiple of four entries
          const int d = 8 * v + 4 * q;
          if (d < 2 * p.pairs) {
            const bool first = d < p.pairs;
            const float4 o = *reinterpret_cast<const float4*>(xbuf + 8 * V * y + (first ? d + p.pairs : d - p.pairs));
            const float2* cs = trig + row_at[i] * p.pairs + (first ? d : d - p.pairs);
            const float other[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float2 t = cs[j];
              x[i][4 * q + j] = x[i][4 * q + j] * t.x + (first ? -other[j] : other[j]) * t.y;
            }
          }
        }
      }
      store8(reinterpret_cast<TOUT*>(side[i]->out) + out[i], x[i]);
    }
    if constexpr (ROT == ROT_HALVES)
      if (i + 1 < ITER) __syncthreads();
  }
}

template <typename TIN, typename TOUT, int NORM, int ROT>
cudaError_t launch(const HeadsParams& p, int D, cudaStream_t st) {
  const int V = D / 8, HB = NTHREADS / V;
  const long long blocks = (p.items + HB * ITER - 1) / (HB * ITER);
  if (blocks > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  const int rows = (HB * ITER - 1) / p.heads + 2;         // a block's items touch no more rows
  const size_t smem = (size_t)((HB * V + 1) & ~1) * sizeof(float2) + (ROT == ROT_HALVES ? (size_t)HB * V * 32 : 0) +
                      (ROT != ROT_NONE ? (size_t)rows * p.pairs * sizeof(float2) : 0);
  cudaLaunchConfig_t lc = {};
  lc.gridDim = dim3((unsigned)blocks); lc.blockDim = dim3((unsigned)V, (unsigned)HB); lc.dynamicSmemBytes = smem; lc.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  lc.attrs = at; lc.numAttrs = g_lq_overlap ? 1 : 0;
  return cudaLaunchKernelEx(&lc, lq_heads_kernel<TIN, TOUT, NORM, ROT>, p);
}
template <typename TIN, typename TOUT, int NORM>
cudaError_t launch_rot(const HeadsParams& p, int D, int rot, cudaStream_t st) {
  return rot == ROT_NONE ? launch<TIN, TOUT, NORM, ROT_NONE>(p, D, st)
         : rot == ROT_PAIRS ? launch<TIN, TOUT, NORM, ROT_PAIRS>(p, D, st) : launch<TIN, TOUT, NORM, ROT_HALVES>(p, D, st);
}
template <typename TIN, typename TOUT>
cudaError_t launch_norm(const HeadsParams& p, int D, int norm, int rot, cudaStream_t st) {
  return norm == LQ_NORM_NONE ? launch_rot<TIN, TOUT, LQ_NORM_NONE>(p, D, rot, st)
         : norm == LQ_NORM_RMS ? launch_rot<TIN, TOUT, LQ_NORM_RMS>(p, D, rot, st) : launch_rot<TIN, TOUT, LQ_NORM_LAYER>(p, D, rot, st);
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
  p.items = rows * p.heads;
  p.seq_len = seq_len; p.axes = R->axes; p.pairs = R->pairs;
  p.eps = eps; p.inv_d = 1.f / (float)head_dim;
  p.turn = R->d_turn; p.axis = R->d_axis; p.pos = pos;
  LqDeviceGuard guard(R->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  const int rot = R->pairs == 0 ? ROT_NONE : R->halves ? ROT_HALVES : ROT_PAIRS;
  cudaStream_t st = (cudaStream_t)stream;
  const cudaError_t e =
      in_dtype == LQ_OUT_F16 ? (out_dtype == LQ_OUT_F16 ? launch_norm<__half, __half>(p, head_dim, norm, rot, st) : launch_norm<__half, float>(p, head_dim, norm, rot, st))
                             : (out_dtype == LQ_OUT_F16 ? launch_norm<float, __half>(p, head_dim, norm, rot, st) : launch_norm<float, float>(p, head_dim, norm, rot, st));
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
