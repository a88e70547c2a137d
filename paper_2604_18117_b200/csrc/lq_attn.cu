// Attention over the cache, the form for few rows (and for heads above 128 entries): one pass over the codes with the running maximum and sum
// of the softmax.
//
//   out = sum_j w_j v_j / sum_j w_j,   w_j = 2^(s_j - max s),   s_j = q . k_j * scale * log2 e,   j over the tokens that the row sees
//
// What bounds it is the memory: a code is read once for all query heads of its group.  The records of all (sequence, head, tile of 16 rows)
// that a launch has lie in a row, tile after tile, and are shared out evenly, neighbouring ones to a block of the grid, so a long sequence
// takes many blocks and ragged batches leave none idle.  A tile whose records are two blocks' or more leaves partial results (unscaled sums,
// maximum, sum), which the last of them to arrive joins in the order of the blocks: no result depends on who was last.
//
// Within a block each warp takes every WARPS-th record, through a ring of its own in shared memory that bulk copies fill.  A record is opened to halves in
// registers (a byte permutation and a packed subtraction for two codes) in the order of m16n8k16 operands; rows' weights go from the
// accumulators of the first product to the operand of the second without a change of lanes.  Weights are rounded to halves there (2^-11 of
// each); sums, maxima and accumulators are fp32.
#include <math.h>

#include "lq_attn.h"
#include "lq_device.cuh"
#include "lq_heads_places.h"

using namespace lqdev;

namespace {

constexpr int ROWS = LQ_ATTN_ROWS;

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Where a record lies in the launch's row of records: walks forward through the sequences that the launch takes.
struct Place {
  LqSeq q;
  LqSeen seen;
  int s, tiles, each;                    // tiles: of rows of the sequence; each: records of a tile
  long long begin, end;                  // of the sequence's records
};
__device__ __forceinline__ void measure(const LqAttnParams& p, int s, Place& at, bool tell) {
  at.s = s;
  at.q = lq_seq(p.b, s);
  at.tiles = at.each = 0;
  if (!lq_attn_takes(p, at.q, tell)) return;
  at.seen = lq_seen(p, at.q.len - at.q.n, at.q.len - 1, at.q.len);
  at.each = max(1, at.seen.count());
  at.tiles = (int)(((long long)at.q.n * p.group + ROWS - 1) / ROWS);
}
__device__ __forceinline__ long long records_of(const LqAttnParams& p, const Place& at) { return (long long)at.tiles * at.each * p.b.heads; }
__device__ __forceinline__ void seek(const LqAttnParams& p, Place& at, long long f) {
  while (f >= at.end && at.s + 1 < p.b.sequences) {
    measure(p, at.s + 1, at, false);
    at.begin = at.end;
    at.end += records_of(p, at);
  }
}

template <int NK, int WARPS, int STAGES>
struct Shared {
  static constexpr int DP = 16 * NK, REC = LQ_KV_HEAD + 2 * LQ_KV_BLOCK * DP, PITCH = DP + 4;
  alignas(16) uint8_t ring[WARPS][STAGES][REC];
  alignas(16) float sums[WARPS][ROWS][PITCH];
  float top[WARPS][ROWS], total[WARPS][ROWS];
  alignas(16) uint32_t q[NK > 8 ? NK : 1][32][4];
  long long prefix[32 * WARPS + 1];
  alignas(8) uint64_t bars[WARPS][STAGES];
  uint8_t empty[WARPS][STAGES];
  int abort_flag, last;
};

template <int NK, int WARPS, int STAGES>
__global__ void __launch_bounds__(32 * WARPS, 1) lq_attn_kernel(const __grid_constant__ LqAttnParams p) {
  using Smem = Shared<NK, WARPS, STAGES>;
  constexpr int DP = 16 * NK, REC = Smem::REC, THREADS = 32 * WARPS;
  extern __shared__ __align__(128) uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c8 = lane >> 2, t = lane & 3;
  if (tid == 0) sm.abort_flag = 0;
  if (lane == 0)
    for (int i = 0; i < STAGES; ++i) mbar_init(smem_u32(&sm.bars[warp][i]), 1);
  mbar_init_fence();
  grid_launch_dependents();
  grid_dependency_wait();

  // the launch's records, and this block's share
  {
    const int chunk = (p.b.sequences + THREADS - 1) / THREADS;
    long long sum = 0;
    for (int s = tid * chunk; s < min(p.b.sequences, (tid + 1) * chunk); ++s) {
      Place at;
      measure(p, s, at, blockIdx.x == 0);
      sum += records_of(p, at);
    }
    long long up = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const long long v = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += v;
    }
    if (lane == 31) sm.prefix[warp] = up;
    __syncthreads();
    long long base = 0;
    for (int i = 0; i < warp; ++i) base += sm.prefix[i];
    __syncthreads();
    sm.prefix[tid + 1] = base + up;
    if (tid == 0) sm.prefix[0] = 0;
    __syncthreads();
  }
  const long long total = sm.prefix[THREADS];
  // at least a record for each warp
  const long long share = max((long long)WARPS, (total + gridDim.x - 1) / gridDim.x);
  const long long lo = blockIdx.x * share, hi = min(total, lo + share);
  if (lo >= hi) return;
  Place here;
  {
    int a = 0, b = THREADS;                                // the last chunk that begins at or before lo
    while (b - a > 1) {
      const int m = (a + b) / 2;
      if (sm.prefix[m] <= lo) a = m; else b = m;
    }
    const int chunk = (p.b.sequences + THREADS - 1) / THREADS;
    measure(p, a * chunk, here, false);
    here.begin = sm.prefix[a];
    here.end = here.begin + records_of(p, here);
    seek(p, here, lo);
  }

  // The warp's ring: record lo + warp, lo + warp + WARPS, ...
  Place ahead = here;
  long long f_ahead = lo + warp;
  int issued = 0;
  const auto issue = [&]() {                               // (a record that is no page's, or of no token, is not fetched; its stage then stays empty)
    if (f_ahead < hi) {
      seek(p, ahead, f_ahead);
      const int i = (int)((f_ahead - ahead.begin) % ahead.each), h = (int)((f_ahead - ahead.begin) / ahead.each / ahead.tiles);
      long long at = -1;
      if (i < ahead.seen.count()) {
        at = lq_kv_at(p.b, ahead.s, ahead.seen.block(i));
        if (at < 0 && lane == 0) lq_kv_refuse(p.status);
      }
      if (lane == 0) {
        const int st = issued % STAGES;
        const uint32_t bar = smem_u32(&sm.bars[warp][st]);
        sm.empty[warp][st] = at < 0;
        if (at >= 0) {
          mbar_expect_tx(bar, REC);
          bulk_load(smem_u32(sm.ring[warp][st]), p.records + (at + h) * p.b.record, REC, bar);
        } else {
          mbar_arrive(bar);
        }
      }
      ++issued;
    }
    f_ahead += WARPS;
  };
  for (int i = 0; i < STAGES; ++i) issue();

  int taken = 0;
  bool good = true;
  long long f = lo + warp;
  for (long long seg = lo; seg < hi;) {
    // a tile of rows, or the part of it that is this block's
    seek(p, here, seg);
    const long long off = seg - here.begin;
    const int tile_no = (int)(off / here.each), h = tile_no / here.tiles, tile = tile_no - h * here.tiles;
    const long long tile_begin = here.begin + (long long)tile_no * here.each, tile_end = tile_begin + here.each;
    const long long seg_end = min(hi, tile_end);
    const int rows = min(ROWS, here.q.n * p.group - tile * ROWS), base = here.q.len - here.q.n;
    // the lane's two rows: c8 and c8 + 8
    int pos[2];
    uint32_t qa[NK > 8 ? 1 : NK][4];
    {
      const __half* from[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = min(tile * ROWS + c8 + 8 * i, here.q.n * p.group - 1), tok = r / p.group;
        pos[i] = base + tok;
        from[i] = p.q + (here.q.row + tok) * p.q_row + (long long)(h * p.group + r - tok * p.group) * p.q_head;
      }
      if (NK <= 8 || warp == 0)
#pragma unroll
        for (int g = 0; g < NK; ++g) {
          uint2 v[2] = {};
          if (16 * g + 4 * t < p.D)
#pragma unroll
            for (int i = 0; i < 2; ++i) v[i] = *reinterpret_cast<const uint2*>(from[i] + 16 * g + 4 * t);
          if constexpr (NK <= 8) {
            qa[g][0] = v[0].x; qa[g][1] = v[1].x; qa[g][2] = v[0].y; qa[g][3] = v[1].y;
          } else {
            *reinterpret_cast<uint4*>(sm.q[g][lane]) = make_uint4(v[0].x, v[1].x, v[0].y, v[1].y);
          }
        }
      if constexpr (NK > 8) __syncthreads();
    }
    const int first_at = base + tile * ROWS / p.group, last_at = base + (tile * ROWS + rows - 1) / p.group;
    float o[NK][2][4] = {};
    float top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
    for (; f < seg_end; f += WARPS) {
      const int st = taken % STAGES;
      if (good) good = mbar_wait_warp(smem_u32(&sm.bars[warp][st]), (taken / STAGES) & 1, &sm.abort_flag, p.status, LQ_STAGE_DRAIN);
      if (!good) break;
      ++taken;
      const uint8_t* rec = sm.ring[warp][st];
      const int i = (int)(f - tile_begin);
      const uint4* ku = reinterpret_cast<const uint4*>(rec + LQ_KV_HEAD) + lane;
      const uint4* vu = ku + 2 * DP;
      const uint32_t tail = *reinterpret_cast<const uint32_t*>(rec);
      const bool empty = sm.empty[warp][st] != 0;
      const int token0 = here.seen.block(i) * LQ_KV_BLOCK;
      if (!empty) {
        float s[4][4] = {};
        {
          const uint32_t high = lq_kv_high((int8_t)(tail & 0xFF));
          const __half2 less = lq_kv_less(high);
#pragma unroll
          for (int g = 0; g < NK; ++g) {
            const uint4 w = ku[32 * g];
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
            uint32_t a[4];
            if constexpr (NK <= 8) {
#pragma unroll
              for (int j = 0; j < 4; ++j) a[j] = qa[g][j];
            } else {
              const uint4 v = *reinterpret_cast<const uint4*>(sm.q[g][lane]);
              a[0] = v.x; a[1] = v.y; a[2] = v.z; a[3] = v.w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) mma_f16(s[j], a, lq_kv_open<0x4140>(ww[j], high, less), lq_kv_open<0x4342>(ww[j], high, less));
          }
        }
        // tile j, column 2 t + b
        const bool all = lq_all_seen(p, first_at, last_at, token0, token0 + LQ_KV_BLOCK - 1, here.q.len);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            const int token = token0 + lq_kv_token(2 * t + b, j);
#pragma unroll
            for (int r = 0; r < 2; ++r) {
              float& x = s[j][2 * r + b];
              x *= p.scale;
              if (!all && !lq_sees(p, pos[r], token, here.q.len)) x = -INFINITY;
            }
          }
        uint32_t w[4][2];                                  // weights of tile j, rows c8 and c8 + 8
        float keep[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          float m = top[r];
#pragma unroll
          for (int j = 0; j < 4; ++j) m = fmaxf(m, fmaxf(s[j][2 * r], s[j][2 * r + 1]));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
          m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
          const float ref = m == -INFINITY ? 0.f : m;      // (a row that has seen nothing yet)
          keep[r] = exp2f(top[r] - ref);
          top[r] = m;
          float add = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float x = exp2f(s[j][2 * r] - ref), y = exp2f(s[j][2 * r + 1] - ref);
            add += x + y;
            w[j][r] = pack(x, y);
          }
          sum[r] = fmaf(sum[r], keep[r], add);
        }
        if (__any_sync(0xffffffffu, keep[0] != 1.f || keep[1] != 1.f)) {
#pragma unroll
          for (int g = 0; g < NK; ++g)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              o[g][j][0] *= keep[0]; o[g][j][1] *= keep[0];
              o[g][j][2] *= keep[1]; o[g][j][3] *= keep[1];
            }
        }
        const uint32_t high = lq_kv_high((int8_t)(tail >> 8 & 0xFF));
        const __half2 less = lq_kv_less(high);
        // tile 2 s, columns 2 t and 2 t + 1: tokens 0 and 2 of the lane's four; tile 2 s + 1: tokens 1 and 3
        const uint32_t a0[4] = {w[0][0], w[0][1], w[1][0], w[1][1]}, a1[4] = {w[2][0], w[2][1], w[3][0], w[3][1]};
#pragma unroll
        for (int g = 0; g < NK; ++g) {
          const uint4 v = vu[32 * g];
          mma_f16(o[g][0], a0, lq_kv_open<0x4240>(v.x, high, less), lq_kv_open<0x4341>(v.x, high, less));
          mma_f16(o[g][1], a0, lq_kv_open<0x4240>(v.y, high, less), lq_kv_open<0x4341>(v.y, high, less));
          mma_f16(o[g][0], a1, lq_kv_open<0x4240>(v.z, high, less), lq_kv_open<0x4341>(v.z, high, less));
          mma_f16(o[g][1], a1, lq_kv_open<0x4240>(v.w, high, less), lq_kv_open<0x4341>(v.w, high, less));
        }
      }
      fence_proxy_async();                                 // the stage is read by all lanes before a copy into it is asked for
      __syncwarp();
      issue();
    }
    // the warps' results of the tile
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 1);
      sum[r] += __shfl_xor_sync(0xffffffffu, sum[r], 2);
      const int row = c8 + 8 * r;
      if (row < rows) {
        if (t == 0) { sm.top[warp][row] = top[r]; sm.total[warp][row] = sum[r]; }
        if (top[r] != -INFINITY)
#pragma unroll
          for (int g = 0; g < NK; ++g)                     // column 2 t + b of tile i is entry 2 (2 t + b) + i of the 16
            *reinterpret_cast<float4*>(&sm.sums[warp][row][16 * g + 4 * t]) = make_float4(o[g][0][2 * r], o[g][1][2 * r], o[g][0][2 * r + 1], o[g][1][2 * r + 1]);
      }
    }
    __syncthreads();
    const bool whole = tile_begin >= lo && tile_end <= hi;
    const long long row0 = (long long)tile * ROWS;
    const auto put = [&](int row, int d, float4 x, float total_w) {
      // values were opened as 2^-4 of themselves
      const float by = total_w > 0.f ? 16.f / total_w : 0.f;
      if (d >= p.D) return;
      const int r = (int)row0 + row, tok = r / p.group;
      __half* to = p.out + (here.q.row + tok) * p.out_row + (long long)(h * p.group + r - tok * p.group) * p.out_head + d;
      *reinterpret_cast<uint2*>(to) = make_uint2(pack(x.x * by, x.y * by), pack(x.z * by, x.w * by));
    };
    const int slot = 2 * blockIdx.x + (tile_begin >= lo ? 1 : 0);
    float* part = p.part + (long long)slot * ROWS * (DP + 2);
    for (int e = tid; e < rows * (DP / 4); e += THREADS) {
      const int row = e / (DP / 4), d = 4 * (e - row * (DP / 4));
      float m = -INFINITY, n = 0.f;
      for (int i = 0; i < WARPS; ++i) m = fmaxf(m, sm.top[i][row]);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int i = 0; i < WARPS; ++i) {
        if (sm.top[i][row] == -INFINITY) continue;
        const float k = exp2f(sm.top[i][row] - m);
        const float4 v = *reinterpret_cast<const float4*>(&sm.sums[i][row][d]);
        n = fmaf(k, sm.total[i][row], n);
        x.x = fmaf(k, v.x, x.x); x.y = fmaf(k, v.y, x.y); x.z = fmaf(k, v.z, x.z); x.w = fmaf(k, v.w, x.w);
      }
      if (whole) {
        put(row, d, x, n);
      } else {
        float* to = part + row * (DP + 2) + 2;
        *reinterpret_cast<float2*>(to + d) = make_float2(x.x, x.y);
        *reinterpret_cast<float2*>(to + d + 2) = make_float2(x.z, x.w);
        if (d == 0) { to[-2] = m; to[-1] = n; }
      }
    }
    if (!whole) {
      const int from = (int)(tile_begin / share), to = (int)((tile_end - 1) / share);
      __threadfence();
      __syncthreads();
      if (tid == 0) {
        const int before = atomicAdd(&p.count[from], 1);
        sm.last = before == to - from;
        if (sm.last) p.count[from] = 0;                    // (nobody else comes)
        __threadfence();
      }
      __syncthreads();
      if (sm.last) {
        for (int e = tid; e < rows * (DP / 4); e += THREADS) {
          const int row = e / (DP / 4), d = 4 * (e - row * (DP / 4));
          const auto of = [&](int c) { return p.part + ((long long)(2 * c + (c == from ? 1 : 0)) * ROWS + row) * (DP + 2); };
          float m = -INFINITY, n = 0.f;
          for (int c = from; c <= to; ++c) m = fmaxf(m, __ldcg(of(c)));
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int c = from; c <= to; ++c) {
            const float* v = of(c);
            const float2 head = __ldcg(reinterpret_cast<const float2*>(v)), u0 = __ldcg(reinterpret_cast<const float2*>(v + 2 + d)),
                         u1 = __ldcg(reinterpret_cast<const float2*>(v + 4 + d));
            if (head.x == -INFINITY) continue;
            const float k = exp2f(head.x - m);
            n = fmaf(k, head.y, n);
            x.x = fmaf(k, u0.x, x.x); x.y = fmaf(k, u0.y, x.y); x.z = fmaf(k, u1.x, x.z); x.w = fmaf(k, u1.y, x.w);
          }
          put(row, d, x, n);
        }
      }
    }
    __syncthreads();                                       // the warps' results are read
    seg = seg_end;
  }
  // (only after a wait that gave up: what is in flight lands before the block leaves)
  if (!good)
    for (; taken < issued; ++taken) mbar_settle(smem_u32(&sm.bars[warp][taken % STAGES]), (taken / STAGES) & 1);
}

// Shared memory holds two to four records of every warp and the warps' sums: eight warps up to 128 entries, four above.
template <int NK, int WARPS, int STAGES>
cudaError_t launch_one(const lq_kvcache* C, const LqAttnParams& p, cudaStream_t st) {
  return lq_launch(lq_attn_kernel<NK, WARPS, STAGES>, C->sms, 32 * WARPS, sizeof(Shared<NK, WARPS, STAGES>), st, p);
}
template <int NK, int WARPS, int STAGES>
bool room() {
  return lq_note_cuda(cudaFuncSetAttribute(lq_attn_kernel<NK, WARPS, STAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                           (int)sizeof(Shared<NK, WARPS, STAGES>))) == cudaSuccess;
}
cudaError_t launch_few(const lq_kvcache* C, const LqAttnParams& p, cudaStream_t st) {
  switch (C->Dp) {
    case 64: return launch_one<4, 8, 4>(C, p, st);
    case 80: return launch_one<5, 8, 3>(C, p, st);
    case 96: return launch_one<6, 8, 2>(C, p, st);
    case 112: return launch_one<7, 8, 2>(C, p, st);
    case 128: return launch_one<8, 8, 2>(C, p, st);
    case 192: return launch_one<12, 4, 3>(C, p, st);
    default: return launch_one<16, 4, 2>(C, p, st);
  }
}

}  // namespace

lq_status lq_attn_prepare(const lq_kvcache* C) {
  const bool ok = C->Dp == 64 ? room<4, 8, 4>() : C->Dp == 80 ? room<5, 8, 3>() : C->Dp == 96 ? room<6, 8, 2>() : C->Dp == 112 ? room<7, 8, 2>()
                  : C->Dp == 128 ? room<8, 8, 2>() : C->Dp == 192 ? room<12, 4, 3>() : room<16, 4, 2>();
  if (!ok) return LQ_ERR_CUDA;
  return C->Dp <= 128 ? lq_attn_tile_prepare(C) : LQ_OK;
}

extern "C" lq_status lq_cache_attention(const lq_kvcache* C, int32_t layer, const lq_kvbatch* batch, const lq_attn* a, void* stream) {
  LqAttnParams p = {};
  lq_status s;
  if (!a) return LQ_ERR_INVALID_ARG;
  if ((s = lq_take_batch(C, layer, batch, &p.b)) != LQ_OK) return s;
  if (!a->q || !a->out || a->q_heads < 1 || a->q_heads % C->heads != 0) return LQ_ERR_INVALID_ARG;
  if ((a->causal != 0 && a->causal != 1) || a->window < 0 || a->sinks < 0) return LQ_ERR_INVALID_ARG;
  if ((a->window > 0 && !a->causal) || (a->sinks > 0 && a->window == 0)) return LQ_ERR_INVALID_ARG;
  if (!(fabsf(a->scale) < 0x1p64f)) return LQ_ERR_INVALID_ARG;
  if (a->q_heads > 4096) return LQ_ERR_UNSUPPORTED;
  if ((((uintptr_t)a->q | (uintptr_t)a->out) & 15) != 0) return LQ_ERR_INVALID_ARG;
  for (int64_t v : {a->q_row, a->q_head, a->out_row, a->out_head}) {
    if (v % 8 != 0) return LQ_ERR_INVALID_ARG;
    if (v >= (1ll << 40) || v <= -(1ll << 40)) return LQ_ERR_UNSUPPORTED;
  }
  if (p.b.rows == 0) return LQ_OK;
  // rows * group and a tile's first row are whole numbers of 32 bits
  if ((long long)p.b.rows * (a->q_heads / C->heads) > (1ll << 30) || (long long)p.b.rows * a->q_heads > (1ll << 34)) return LQ_ERR_UNSUPPORTED;
  const LqRuns q{(uintptr_t)a->q, {2 * a->q_row, 2 * a->q_head, 0}, {p.b.rows, a->q_heads, 1}, 2ll * C->D};
  const LqRuns out{(uintptr_t)a->out, {2 * a->out_row, 2 * a->out_head, 0}, {p.b.rows, a->q_heads, 1}, 2ll * C->D};
  const auto status = [](LqPlaces c) { return c == LQ_APART ? LQ_OK : c == LQ_SHARED ? LQ_ERR_INVALID_ARG : LQ_ERR_UNSUPPORTED; };
  if ((s = status(lq_runs_collide(out))) != LQ_OK || (s = status(lq_runs_meet(out, q))) != LQ_OK) return s;
  LqDeviceGuard guard(C->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  p.records = lq_kv_layer(C, layer);
  p.q = (const __half*)a->q; p.out = (__half*)a->out;
  p.q_row = a->q_row; p.q_head = a->q_head; p.out_row = a->out_row; p.out_head = a->out_head;
  p.D = C->D; p.Dp = C->Dp; p.group = a->q_heads / C->heads;
  p.causal = a->causal; p.window = a->window; p.sinks = a->sinks;
  p.scale = a->scale * 16.f * 1.44269504088896341f;        // (keys are opened as 2^-4 of themselves)
  p.part = C->d_part; p.count = C->d_count;
  p.status = lq_device_status_ptr(C->device);
  // Which form a sequence's rows are the kernels tell by themselves where sequences have different numbers of them; a form that no sequence can be is
  // not launched.
  const bool tiles = C->Dp <= 128;
  const long long most = p.b.row_start ? (long long)p.b.rows * p.group : (long long)p.b.each * p.group, least = p.b.row_start ? 1 : most;
  if (!tiles || least <= LQ_ATTN_FEW) {
    p.few = 1;
    p.many = tiles ? LQ_ATTN_FEW + 1 : 0x7fffffff;
    if (lq_note_cuda(launch_few(C, p, (cudaStream_t)stream)) != cudaSuccess) return LQ_ERR_CUDA;
  }
  if (tiles && most > LQ_ATTN_FEW) {
    p.few = LQ_ATTN_FEW + 1;
    p.many = 0x7fffffff;
    return lq_attn_tile_launch(C, p, (cudaStream_t)stream);
  }
  return LQ_OK;
}
