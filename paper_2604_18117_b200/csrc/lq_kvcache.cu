// A paged cache of keys and values in 8 bits: quantised as it is written, and read back.
//
//   a block of 32 tokens of a head has one step 2^e for its keys and one for its values, e the smallest integer in [-20, 9] with
//   127 * 2^e >= the largest magnitude that was written to it;   code c = rint(x / 2^e) in [-127, 127]
//
// Tokens that come to a block that has some already may need a larger e'; the codes that are there become rint(c / 2^(e' - e)).  Powers of two
// make both divisions exact, and every value c 2^e is a half (of 11 bits: c has 7).
#include <math.h>

#include <algorithm>
#include <new>

#include "lq_device.cuh"
#include "lq_heads_places.h"
#include "lq_kvcache.h"

using namespace lqdev;

namespace {

constexpr int WARPS = 4;

struct RowsParams {
  LqBatch b;
  uint8_t* records;
  void *k, *v;
  long long seq[2], row[2], head[2];     // strides in elements
  int D, Dp, tile;                       // tile: rows that a warp looks through
  const int32_t* begin;
  int most, blocks;                      // read: most tokens of a sequence, blocks that they can touch
  int32_t* status;
};

template <typename T>
__device__ __forceinline__ float4 load4(const T* p);
template <>
__device__ __forceinline__ float4 load4<float>(const float* p) { return *reinterpret_cast<const float4*>(p); }
template <>
__device__ __forceinline__ float4 load4<__half>(const __half* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
  return make_float4(a.x, a.y, b.x, b.y);
}
template <typename T>
__device__ __forceinline__ float2 load2(const T* p);
template <>
__device__ __forceinline__ float2 load2<float>(const float* p) { return *reinterpret_cast<const float2*>(p); }
template <>
__device__ __forceinline__ float2 load2<__half>(const __half* p) { return __half22float2(*reinterpret_cast<const __half2*>(p)); }

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
// smallest e in range with 127 * 2^e >= top
__device__ __forceinline__ int exponent_of(float top) {
  const uint32_t bits = __float_as_uint(top);
  // top = (1 + m) 2^x: 127 * 2^(x - 6) = (1 + 63 / 64) 2^x
  const int x = (int)(bits >> 23) - 127, e = x - 6 + ((bits & 0x7FFFFF) > (63u << 17));
  return max(LQ_KV_E_MIN, min(LQ_KV_E_MAX, e));
}
__device__ __forceinline__ uint32_t code_of(float x, float inv) {         // byte c + 128
  return (uint32_t)(__float2int_rn(fminf(fmaxf(x * inv, -127.f), 127.f)) + 128);
}
// rint(c / 2^k) of a byte c + 128
__device__ __forceinline__ uint32_t shrink(uint32_t u, float inv) { return (uint32_t)(__float2int_rn((float)((int)u - 128) * inv) + 128); }

// The sequence that row r belongs to: the last one that begins at or before it and has rows, found by the warp together.
__device__ __forceinline__ int sequence_of(const LqBatch& b, int r, int lane) {
  if (!b.row_start) return r / b.each;
  int lo = 0, n = b.sequences;           // the answer is in [lo, lo + n)
  while (n > 1) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const bool before = at < lo + n && b.row_start[at] <= r;
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, before) | 1);
    lo += last * step;
    n = min(step, n - last * step);
  }
  return lo;
}

// One block, keys or values, one warp: tokens t0 .. t1 - 1 of it are new, rows of `in` from that of t0 on; those before t0 are there already.
template <typename T, bool KEYS>
__device__ void write_block(uint8_t* record, const T* in, long long row, int t0, int t1, int D, int Dp, int lane) {
  const int chunks = D / 8, n = t1 - t0;
  float top = 0.f;
  for (int i = lane; i < n * chunks; i += 32) {
    const int r = i / chunks, c = i - r * chunks;
    const T* p = in + r * row + 8 * c;
    const float4 a = load4(p), b = load4(p + 4);
    top = fmaxf(top, fmaxf(fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(a.z), fabsf(a.w))), fmaxf(fmaxf(fabsf(b.x), fabsf(b.y)), fmaxf(fabsf(b.z), fabsf(b.w)))));
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  int8_t* exps = reinterpret_cast<int8_t*>(record) + (KEYS ? 0 : 1);
  const int need = exponent_of(top), was = t0 > 0 ? max(LQ_KV_E_MIN, min(LQ_KV_E_MAX, (int)*exps)) : LQ_KV_E_MIN, e = max(need, was);
  const bool grows = t0 > 0 && e > was;
  const float inv = pow2(-e), less = pow2(was - e);
  __syncwarp();
  if (lane == 0) *exps = (int8_t)e;
  uint8_t* side = record + LQ_KV_HEAD + (KEYS ? 0 : lq_kv_side_bytes(Dp));
  const int c8 = lane >> 2, t = lane & 3;
  // Bit i: the lane's unit has token i of the block.  Units without a token to write are left alone.
  const uint32_t mine = KEYS ? 0x00030003u << (2 * c8) : 0x000F000Fu << (4 * t);
  const uint32_t below1 = t1 == 32 ? 0xffffffffu : (1u << t1) - 1, fresh = below1 & ~((1u << t0) - 1);
  if (!(mine & (grows ? below1 : fresh))) return;
  const bool keeps = t0 > 0 && (mine & ((1u << t0) - 1)) != 0;
  for (int g = 0; g < Dp / 16; ++g) {
    uint4* at = reinterpret_cast<uint4*>(side + 512 * g + 16 * lane);
    uint32_t w[4] = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};
    if (keeps) {
      const uint4 v = *at;
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
      if (grows)                         // (what lies behind the old tokens is written below, or is no token's)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          w[i] = shrink(w[i] & 0xFF, less) | shrink((w[i] >> 8) & 0xFF, less) << 8 | shrink((w[i] >> 16) & 0xFF, less) << 16 | shrink(w[i] >> 24, less) << 24;
    }
    if constexpr (KEYS) {
      const int d = 16 * g + 4 * t;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int token = lq_kv_token(c8, i);
        if (token < t0 || token >= t1) continue;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (d < D) x = load4(in + (token - t0) * row + d);
        w[i] = code_of(x.x, inv) | code_of(x.y, inv) << 8 | code_of(x.z, inv) << 16 | code_of(x.w, inv) << 24;
      }
    } else {
      const int d = 16 * g + 2 * c8;
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int token = 16 * s + 4 * t + i;
          if (token < t0 || token >= t1) continue;
          float2 x = make_float2(0.f, 0.f);
          if (d < D) x = load2(in + (token - t0) * row + d);
          w[2 * s] = (w[2 * s] & ~(0xFFu << (8 * i))) | code_of(x.x, inv) << (8 * i);
          w[2 * s + 1] = (w[2 * s + 1] & ~(0xFFu << (8 * i))) | code_of(x.y, inv) << (8 * i);
        }
    }
    *at = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// A warp takes a head's keys or values in the blocks that begin within its tile of rows: with a sequence's first new row, or with a token
// that is the first of its block.
template <typename T>
__global__ void __launch_bounds__(32 * WARPS) lq_kv_append_kernel(const __grid_constant__ RowsParams p) {
  const int lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
  grid_launch_dependents();
  grid_dependency_wait();
  const int side = (int)(task & 1);
  const long long rest = task >> 1;
  const int head = (int)(rest % p.b.heads);
  const long long first = rest / p.b.heads * p.tile;
  if (first >= p.b.rows) return;
  int r = (int)first;
  const int end = (int)min((long long)p.b.rows, first + p.tile);
  const T* in = reinterpret_cast<const T*>(side ? p.v : p.k) + head * p.head[side];
  int s = sequence_of(p.b, r, lane);
  while (r < end && s < p.b.sequences) {
    const LqSeq q = lq_seq(p.b, s);
    if (r < q.row || q.n == 0 || r >= q.row + q.n) {       // rows of no sequence lie in front (then r moves on), or the next sequence has it
      if (r < q.row) r = q.row;
      else ++s;
      continue;
    }
    if (!lq_seq_fits(p.b, q) || q.len < q.n) {
      if (lane == 0) lq_kv_refuse(p.status);
      r = q.row + q.n;
      continue;
    }
    const int at = q.len - q.n + (r - q.row), t0 = at % LQ_KV_BLOCK, t1 = min(LQ_KV_BLOCK, t0 + q.row + q.n - r);
    if (r == q.row || t0 == 0) {
      const long long record = lq_kv_at(p.b, s, at / LQ_KV_BLOCK);
      if (record < 0) {
        if (lane == 0) lq_kv_refuse(p.status);
      } else {
        uint8_t* to = p.records + (record + head) * p.b.record;
        if (side) write_block<T, false>(to, in + r * p.row[side], p.row[side], t0, t1, p.D, p.Dp, lane);
        else write_block<T, true>(to, in + r * p.row[side], p.row[side], t0, t1, p.D, p.Dp, lane);
      }
    }
    r += t1 - t0;
  }
}

template <typename T>
__device__ __forceinline__ void store4(T* p, float4 x);
template <>
__device__ __forceinline__ void store4<float>(float* p, float4 x) { *reinterpret_cast<float4*>(p) = x; }
template <>
__device__ __forceinline__ void store4<__half>(__half* p, float4 x) {
  const __half2 a = __floats2half2_rn(x.x, x.y), b = __floats2half2_rn(x.z, x.w);
  *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}
template <typename T>
__device__ __forceinline__ void store2(T* p, float x, float y);
template <>
__device__ __forceinline__ void store2<float>(float* p, float x, float y) { *reinterpret_cast<float2*>(p) = make_float2(x, y); }
template <>
__device__ __forceinline__ void store2<__half>(__half* p, float x, float y) { *reinterpret_cast<__half2*>(p) = __floats2half2_rn(x, y); }

__device__ __forceinline__ float value_of(uint32_t w, int i, float step) { return (float)((int)((w >> (8 * i)) & 0xFF) - 128) * step; }

// A warp takes a head's keys or values of one block.
template <typename T>
__global__ void __launch_bounds__(32 * WARPS) lq_kv_read_kernel(const __grid_constant__ RowsParams p) {
  const int lane = threadIdx.x & 31;
  const long long task = (long long)blockIdx.x * WARPS + (threadIdx.x >> 5);
  grid_launch_dependents();
  grid_dependency_wait();
  const int side = (int)(task & 1);
  long long rest = task >> 1;
  const int head = (int)(rest % p.b.heads);
  rest /= p.b.heads;
  const int s = (int)(rest / p.blocks), i = (int)(rest % p.blocks);
  if (s >= p.b.sequences || (side ? p.v : p.k) == nullptr) return;
  LqSeq q;
  q.len = p.b.length[s];
  const int begin = p.begin ? p.begin[s] : 0;
  if (!lq_seq_fits(p.b, q) || begin < 0) {
    if (lane == 0) lq_kv_refuse(p.status);
    return;
  }
  const long long block = (long long)begin / LQ_KV_BLOCK + i;
  const int end = (int)min((long long)q.len, (long long)begin + p.most);
  if (block * LQ_KV_BLOCK >= end) return;
  const long long at = lq_kv_at(p.b, s, (int)block);
  if (at < 0) {
    if (lane == 0) lq_kv_refuse(p.status);
    return;
  }
  const uint8_t* record = p.records + (at + head) * p.b.record;
  const int e = reinterpret_cast<const int8_t*>(record)[side];
  const float step = pow2(e);
  const uint4* units = reinterpret_cast<const uint4*>(record + LQ_KV_HEAD + (side ? lq_kv_side_bytes(p.Dp) : 0)) + lane;
  const int c8 = lane >> 2, t = lane & 3, first = (int)(block * LQ_KV_BLOCK);
  T* out = reinterpret_cast<T*>(side ? p.v : p.k) + s * p.seq[side] + head * p.head[side] + ((long long)first - begin) * p.row[side];
  for (int g = 0; 16 * g < p.D; ++g) {
    const uint4 v = units[32 * g];
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (side == 0) {
      const int d = 16 * g + 4 * t;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int token = lq_kv_token(c8, j);
        if (d < p.D && first + token >= begin && first + token < end)
          store4(out + token * p.row[side] + d, make_float4(value_of(w[j], 0, step), value_of(w[j], 1, step), value_of(w[j], 2, step), value_of(w[j], 3, step)));
      }
    } else {
      const int d = 16 * g + 2 * c8;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int token = 16 * (j >> 2) + 4 * t + (j & 3), half = 2 * (j >> 2);
        if (d < p.D && first + token >= begin && first + token < end)
          store2(out + token * p.row[side] + d, value_of(w[half], j & 3, step), value_of(w[half + 1], j & 3, step));
      }
    }
  }
}

// Strides of one side's rows: multiples of 8 elements, so that every head begins on a 16-byte boundary.
lq_status take_rows(const lq_kvrows* r, RowsParams* p) {
  p->k = r->k; p->v = r->v;
  if ((((uintptr_t)r->k | (uintptr_t)r->v) & 15) != 0) return LQ_ERR_INVALID_ARG;
  const int64_t strides[6] = {r->k_seq, r->v_seq, r->k_row, r->v_row, r->k_head, r->v_head};
  for (int64_t v : strides) {
    if (v % 8 != 0) return LQ_ERR_INVALID_ARG;
    if (v >= (1ll << 40) || v <= -(1ll << 40)) return LQ_ERR_UNSUPPORTED;
  }
  for (int i = 0; i < 2; ++i) { p->seq[i] = strides[i]; p->row[i] = strides[2 + i]; p->head[i] = strides[4 + i]; }
  return LQ_OK;
}

}  // namespace

lq_status lq_take_batch(const lq_kvcache* C, int32_t layer, const lq_kvbatch* b, LqBatch* out) {
  if (!C || !b || layer < 0 || layer >= C->layers) return LQ_ERR_INVALID_ARG;
  if (b->sequences < 1 || b->rows < 0 || !b->length || !b->pages || b->page_stride < 1) return LQ_ERR_INVALID_ARG;
  if ((((uintptr_t)b->row_start | (uintptr_t)b->length | (uintptr_t)b->pages) & 3) != 0) return LQ_ERR_INVALID_ARG;
  if (b->sequences > LQ_KV_MAX_SEQUENCES) return LQ_ERR_UNSUPPORTED;
  if (!b->row_start && b->rows % b->sequences != 0) return LQ_ERR_INVALID_ARG;
  *out = LqBatch{b->row_start, b->length, b->pages, b->sequences, b->rows, b->rows / b->sequences, b->page_stride, C->pages, C->page_tokens / LQ_KV_BLOCK,
                 C->heads, lq_kv_record_bytes(C->Dp), ((1ull << 37) + C->page_tokens / LQ_KV_BLOCK - 1) / (C->page_tokens / LQ_KV_BLOCK)};
  return LQ_OK;
}

extern "C" lq_status lq_kvcache_create(int32_t layers, int32_t pages, int32_t page_tokens, int32_t kv_heads, int32_t head_dim, int device,
                                       lq_kvcache** out) {
  if (!out || layers < 1 || pages < 1 || page_tokens < 1 || kv_heads < 1 || head_dim < 1) return LQ_ERR_INVALID_ARG;
  if (page_tokens % LQ_KV_BLOCK != 0 || page_tokens > 65536 || kv_heads > 4096 || head_dim % 8 != 0 || head_dim > 256) return LQ_ERR_UNSUPPORTED;
  const int Dp = lq_kv_padded(head_dim);
  const double records = (double)layers * pages * (page_tokens / LQ_KV_BLOCK) * kv_heads;
  if (records * lq_kv_record_bytes(Dp) > 0x1p46) return LQ_ERR_ALLOC;          // (no such memory; below it sizes are whole numbers of 64 bits)
  int ndev = 0;
  if (lq_note_cuda(cudaGetDeviceCount(&ndev)) != cudaSuccess || device < 0 || device >= ndev) return LQ_ERR_CUDA;
  LqDeviceGuard guard(device);
  if (!guard.ok) return LQ_ERR_CUDA;
  lq_kvcache* C = new (std::nothrow) lq_kvcache();
  if (!C) return LQ_ERR_ALLOC;
  C->layers = layers; C->pages = pages; C->page_tokens = page_tokens; C->heads = kv_heads; C->D = head_dim; C->Dp = Dp; C->device = device;
  const size_t n = (size_t)records, rec = lq_kv_record_bytes(Dp);
  if (lq_note_cuda(cudaDeviceGetAttribute(&C->sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess) {
    lq_kvcache_free(C);
    return LQ_ERR_CUDA;
  }
  if (lq_note_cuda(cudaMalloc((void**)&C->d_records, n * rec)) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&C->d_part, (size_t)2 * C->sms * LQ_ATTN_ROWS * (Dp + 4) * sizeof(float))) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&C->d_count, C->sms * sizeof(int))) != cudaSuccess) {
    lq_kvcache_free(C);
    return LQ_ERR_ALLOC;
  }
  // All zeros (code 0, exponent 0): what no token has been written to is multiplied with zero weights, and has to be a number.
  if (lq_note_cuda(cudaMemset(C->d_records, 0x80, n * rec)) != cudaSuccess ||
      lq_note_cuda(cudaMemset2D(C->d_records, rec, 0, LQ_KV_HEAD, n)) != cudaSuccess ||
      lq_note_cuda(cudaMemset(C->d_count, 0, C->sms * sizeof(int))) != cudaSuccess || lq_note_cuda(cudaDeviceSynchronize()) != cudaSuccess ||
      !lq_device_status_ptr(device)) {                       // (allocated here, not under a capture)
    lq_kvcache_free(C);
    return LQ_ERR_CUDA;
  }
  lq_status s;
  if ((s = lq_attn_prepare(C)) != LQ_OK) {
    lq_kvcache_free(C);
    return s;
  }
  *out = C;
  return LQ_OK;
}

extern "C" lq_status lq_kvcache_free(lq_kvcache* C) {
  if (!C) return LQ_ERR_INVALID_ARG;
  LqDeviceGuard guard(C->device);
  cudaFree(C->d_records); cudaFree(C->d_part); cudaFree(C->d_count);
  delete C;
  return LQ_OK;
}

extern "C" lq_status lq_kvcache_append(lq_kvcache* C, int32_t layer, const lq_kvbatch* batch, const lq_kvrows* rows, lq_out_dtype dt, void* stream) {
  RowsParams p = {};
  lq_status s;
  if (!rows || (dt != LQ_OUT_F16 && dt != LQ_OUT_F32)) return LQ_ERR_INVALID_ARG;
  if ((s = lq_take_batch(C, layer, batch, &p.b)) != LQ_OK || (s = take_rows(rows, &p)) != LQ_OK) return s;
  if (!p.k || !p.v) return LQ_ERR_INVALID_ARG;
  if (p.b.rows == 0) return LQ_OK;
  LqDeviceGuard guard(C->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  p.records = lq_kv_layer(C, layer);
  p.D = C->D; p.Dp = C->Dp;
  p.status = lq_device_status_ptr(C->device);
  // Rows a warp looks through: 32, as many as a block has, once that gives every SM 32 warps; with fewer rows fewer, so that blocks of
  // different sequences are not one warp's.
  const long long tasks = 2ll * C->heads * p.b.rows;
  p.tile = (int)std::max(1ll, std::min(32ll, tasks / (32ll * C->sms)));
  const long long blocks = (2ll * C->heads * lq_ceil_div(p.b.rows, p.tile) + WARPS - 1) / WARPS;
  if (blocks > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  const cudaError_t e = dt == LQ_OUT_F16 ? lq_launch(lq_kv_append_kernel<__half>, (int)blocks, 32 * WARPS, 0, (cudaStream_t)stream, p)
                                         : lq_launch(lq_kv_append_kernel<float>, (int)blocks, 32 * WARPS, 0, (cudaStream_t)stream, p);
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}

extern "C" lq_status lq_kvcache_read(const lq_kvcache* C, int32_t layer, const lq_kvbatch* batch, const int32_t* begin, int32_t most, const lq_kvrows* rows,
                                     lq_out_dtype dt, void* stream) {
  RowsParams p = {};
  lq_status s;
  if (!rows || most < 1 || ((uintptr_t)begin & 3) != 0 || (dt != LQ_OUT_F16 && dt != LQ_OUT_F32)) return LQ_ERR_INVALID_ARG;
  if ((s = lq_take_batch(C, layer, batch, &p.b)) != LQ_OK || (s = take_rows(rows, &p)) != LQ_OK) return s;
  if (!p.k && !p.v) return LQ_ERR_INVALID_ARG;
  p.begin = begin;
  // (no sequence has more tokens than its row of pages)
  p.most = (int)std::min((long long)most, (long long)p.b.page_stride * C->page_tokens);
  p.blocks = (int)(((long long)p.most + 2 * LQ_KV_BLOCK - 2) / LQ_KV_BLOCK);
  // no two entries of the outputs on one place
  LqRuns out[2];
  int n = 0;
  for (int i = 0; i < 2; ++i)
    if (i == 0 ? p.k : p.v) {
      const int64_t esz = dt == LQ_OUT_F32 ? 4 : 2;
      out[n++] = LqRuns{(uintptr_t)(i == 0 ? p.k : p.v), {p.seq[i] * esz, p.row[i] * esz, p.head[i] * esz}, {p.b.sequences, p.most, C->heads}, C->D * esz};
    }
  const auto status = [](LqPlaces c) { return c == LQ_APART ? LQ_OK : c == LQ_SHARED ? LQ_ERR_INVALID_ARG : LQ_ERR_UNSUPPORTED; };
  for (int i = 0; i < n; ++i)
    if ((s = status(lq_runs_collide(out[i]))) != LQ_OK) return s;
  if (n == 2 && (s = status(lq_runs_meet(out[0], out[1]))) != LQ_OK) return s;
  LqDeviceGuard guard(C->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  p.records = lq_kv_layer(C, layer);
  p.D = C->D; p.Dp = C->Dp;
  p.status = lq_device_status_ptr(C->device);
  const long long blocks = (2ll * C->heads * p.b.sequences * p.blocks + WARPS - 1) / WARPS;
  if (blocks > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  const cudaError_t e = dt == LQ_OUT_F16 ? lq_launch(lq_kv_read_kernel<__half>, (int)blocks, 32 * WARPS, 0, (cudaStream_t)stream, p)
                                         : lq_launch(lq_kv_read_kernel<float>, (int)blocks, 32 * WARPS, 0, (cudaStream_t)stream, p);
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
