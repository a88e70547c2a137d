// Attention over the cache, the form for few rows (and for heads above 128 entries): one pass over the codes with the running maximum and sum
// of the softmax.
//
//   out = sum_j w_j v_j / sum_j w_j,   w_j = 2^(s_j - max s),   s_j = q . k_j * scale * log2 e,   j over the tokens that the row sees
//
// What bounds it is the memory: a code is read once for all query heads of its group.  The records of all (sequence, head, tile of 16 rows)
// that a launch has lie in a row, tile after tile, and are shared out evenly, neighbouring ones to a block of the grid, so a long sequence
// takes many blocks and ragged batches leave none idle.  A tile whose records are two blocks' or more leaves partial results (unscaled sums,
// maximum, sum), which the last of them to arrive joins in the order of the blocks: no result depends on who was last.  That costs some 2 us, as
// much as a few records a warp, so a tile of few records is one block's as a whole.
//
// Within a block each warp takes every WARPS-th record, through a ring of its own in shared memory that bulk copies fill.  A record is opened
// to halves in registers (a byte permutation and a packed subtraction for two codes), which are the first operands of m16n8k16 products: S^T =
// K Q^T with 8 or 16 rows of Q as columns, so that no more products are made than rows ask for, and O^T = V^T W^T.  The rows' weights are
// rounded to halves between the two (lq_attn.h says what that keeps of small ones) and turned round 8 x 8 at a time; sums, maxima and accumulators are
// fp32.  Accumulators are only scaled when a row's maximum has grown by 8 or more (in powers of two).
//
// B200, us of passes back to back in graphs and TB/s of the visible codes: one token of 131072, 8 heads of 128, 32 queries 50.4, 5.3 (records stream at
// some 7 TB/s once they do: 4 us of start, 2 to 3 of the join, the rest launch and end); 64 sequences of 1 to 8192 tokens 107.5, 5.0 (the same start
// and joins at three to six tiles a block), with 4 heads of 256 for 16 queries 101, 5.3; 24 times three tokens, window 1000, 2 heads of 80 14.7; one token
// of 300 6.6, a chain of latencies.  Prompts of heads above 128 entries, which have no other form: 2048 tokens of 4096, 16 heads on 4 of 256 931, 111
// TFLOP/s.
// With 16 rows where 8 would do (both products at twice the width) the long sequence took 89 us, with a ring of three, one or 16 warps' records
// the same as with this one.
#include <math.h>

#include "lq_attn.h"
#include "lq_attn_places.h"
#include "lq_device.cuh"
#include "lq_heads_places.h"

using namespace lqdev;

namespace {

constexpr int SHORT = 4;                 // records a warp of a tile that is not shared out

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, const uint2& b) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b.x), "r"(b.y));
}
__device__ __forceinline__ uint32_t turned(uint32_t v) {  // 8 x 8 halves, rows for columns
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ int add_acq_rel(int* p, int v) {
  int before;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(before) : "l"(p), "r"(v) : "memory");
  return before;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

struct Seq {
  LqSeq rows;
  LqSeen seen;
};
using Place = LqAttnPlace<Seq>;
template <int ROWS>
__device__ __forceinline__ Place measure(const LqAttnParams& p, int s, bool tell) {
  Place at = {};
  at.s = s;
  const LqSeq q = at.q.rows = lq_seq(p.b, s);
  if (!lq_attn_takes(p, q, tell)) return at;
  at.q.seen = lq_seen(p, q.len - q.n, q.len - 1, q.len);
  at.each = max(1, at.q.seen.count());
  at.tiles = (int)(((long long)q.n * p.group + ROWS - 1) / ROWS);
  return at;
}

template <int NK, int NT, int WARPS, int STAGES>
struct Shared {
  static constexpr int DP = 16 * NK, REC = LQ_KV_HEAD + 2 * LQ_KV_BLOCK * DP, PITCH = DP + 4, ROWS = 8 * NT;
  static constexpr bool Q_HERE = NK * NT > 16;             // Q in shared memory: its registers would not be there
  alignas(16) uint8_t ring[WARPS][STAGES][REC];
  alignas(16) float sums[WARPS][ROWS][PITCH];
  float top[WARPS][ROWS], total[WARPS][ROWS];
  alignas(16) uint2 q[Q_HERE ? NK : 1][NT][32];
  long long prefix[WARPS], tiles[WARPS], edge[2];
  Place found;
  alignas(8) uint64_t bars[WARPS][STAGES];
  uint8_t empty[WARPS][STAGES];
  int abort_flag, last, part, parts;
};

template <int NK, int NT, int WARPS, int STAGES>
__global__ void __launch_bounds__(32 * WARPS, 1) lq_attn_kernel(const __grid_constant__ LqAttnParams p) {
  using Smem = Shared<NK, NT, WARPS, STAGES>;
  constexpr int DP = 16 * NK, REC = Smem::REC, THREADS = 32 * WARPS, ROWS = 8 * NT;
  extern __shared__ __align__(128) uint8_t raw[];
  Smem& sm = *reinterpret_cast<Smem*>(raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, c8 = lane >> 2, t = lane & 3;
  if (tid == 0) sm.abort_flag = 0;
  if (lane == 0)
    for (int i = 0; i < STAGES; ++i) mbar_init(smem_u32(&sm.bars[warp][i]), 1);
  mbar_init_fence();
  grid_launch_dependents();
  grid_dependency_wait();
  const auto sequence = [&](int s) { return measure<ROWS>(p, s, false); };

  // The launch's records, and this block's share of them: from edge[0] on, a place that is found, to before edge[1].  The thread among whose
  // sequences an edge is looks it up.
  LqAttnCut cut;
  {
    const int chunk = (p.b.sequences + THREADS - 1) / THREADS, first = tid * chunk, behind = min(p.b.sequences, first + chunk);
    Place mine = {};                                       // the thread's first sequence
    long long records = 0, tiles = 0;
    for (int s = first; s < behind; ++s) {
      const Place at = measure<ROWS>(p, s, blockIdx.x == 0);
      if (s == first) mine = at;
      records += lq_attn_records(at, p.b.heads);
      tiles += (long long)at.tiles * p.b.heads;
    }
    long long all = records;
#pragma unroll
    for (int d = 16; d > 0; d /= 2) {
      all += __shfl_xor_sync(0xffffffffu, all, d);
      tiles += __shfl_xor_sync(0xffffffffu, tiles, d);
    }
    if (lane == 0) { sm.prefix[warp] = all; sm.tiles[warp] = tiles; }
    __syncthreads();
    all = tiles = 0;
#pragma unroll
    for (int i = 0; i < WARPS; ++i) { all += sm.prefix[i]; tiles += sm.tiles[i]; }
    cut = lq_attn_cut(all, tiles, gridDim.x, WARPS);
    long long count = records;
    if (cut.parted) {
      count = lq_attn_count(mine, p.b.heads, cut, SHORT * WARPS);
      for (int s = first + 1; s < behind; ++s) count += lq_attn_count(sequence(s), p.b.heads, cut, SHORT * WARPS);
    }
    long long up = count;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const long long v = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += v;
    }
    __syncthreads();
    if (lane == 31) sm.prefix[warp] = up;
    if (tid == 0) { sm.edge[0] = sm.edge[1] = cut.parted ? 0 : all; }
    __syncthreads();
    long long begin = up - count;
    for (int i = 0; i < warp; ++i) begin += sm.prefix[i];
    if (cut.parted) {
      if ((long long)blockIdx.x >= begin && (long long)blockIdx.x < begin + count) {
        Place at = mine;
        sm.edge[1] = lq_attn_part(at, begin, blockIdx.x, p.b.heads, SHORT * WARPS, cut, sm.part, sm.parts, sequence);
        sm.found = at;
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < 2; ++i) {
        const long long edge = (blockIdx.x + i) * cut.share;
        if (edge < begin || edge >= begin + count) continue;
        Place at = mine;
        const long long there = lq_attn_edge(at, begin, edge, p.b.heads, SHORT * WARPS, sequence);
        sm.edge[i] = there;
        if (i == 0) {
          if (there < all) lq_attn_walk(at, 0, p.b.heads, p.b.sequences, sequence);
          sm.found = at;
        }
      }
    }
    __syncthreads();
  }
  const long long lo = sm.edge[0], hi = sm.edge[1];
  if (lo >= hi) return;
  Place here = sm.found;

  const float scale = lq_attn_scale(p);
  uint2 qb[Smem::Q_HERE ? 1 : NK][NT];
  const auto load_q = [&](const Place& at) {
    const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;              // of the signs of Q
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = at.tile * ROWS + 8 * n + c8, tok = r / p.group;
      const bool real = r < at.q.rows.n * p.group;
      const __half* from = p.q + (at.q.rows.row + tok) * p.q_row + (long long)(at.head * p.group + r - tok * p.group) * p.q_head + 4 * t;
#pragma unroll
      for (int g = 0; g < NK; ++g) {
        uint2 v = make_uint2(0, 0);
        if (real && 16 * g + 4 * t < p.D) {
          v = *reinterpret_cast<const uint2*>(from + 16 * g);
          v.x ^= flip; v.y ^= flip;
        }
        if constexpr (Smem::Q_HERE) sm.q[g][n][lane] = v;
        else qb[g][n] = v;
      }
    }
  };
  if constexpr (!Smem::Q_HERE) load_q(here);               // (here and below: asked for ahead of the wait for something else)

  // The warp's ring: records lo + warp, lo + warp + WARPS, ...  Where they lie is looked up for 32 of them at a time, one a lane.
  Place ahead = here;                                      // of the first that has not been looked up
  int left = (int)((hi - lo - warp + WARPS - 1) / WARPS), looked = 0, issued = 0;
  long long mine = -1;                                     // the lane's record, -1: no page's, or of no token
  if (left > 0) lq_attn_walk(ahead, warp, p.b.heads, p.b.sequences, sequence);
  const auto look = [&]() {
    Place at = ahead;
    mine = -1;
    if (lane < left - looked && lq_attn_walk(at, lane * WARPS, p.b.heads, p.b.sequences, sequence) && at.i < at.q.seen.count()) {
      mine = lq_kv_at(p.b, at.s, at.q.seen.block(at.i));
      if (mine < 0) lq_kv_refuse(p.status);
      else mine += at.head;
    }
    __syncwarp();
    looked += 32;
    if (looked < left && !lq_attn_walk(ahead, 32 * WARPS, p.b.heads, p.b.sequences, sequence)) left = looked;
  };
  const auto issue = [&]() {                               // (what is not fetched leaves its stage empty)
    if (issued >= left) return;
    if (issued == looked) look();
    const long long at = __shfl_sync(0xffffffffu, mine, issued & 31);
    if (lane == 0) {
      const int st = issued % STAGES;
      const uint32_t bar = smem_u32(&sm.bars[warp][st]);
      sm.empty[warp][st] = at < 0;
      if (at >= 0) {
        mbar_expect_tx(bar, REC);
        bulk_load(smem_u32(sm.ring[warp][st]), p.records + at * p.b.record, REC, bar);
      } else {
        mbar_arrive(bar);
      }
    }
    ++issued;
  };
  for (int i = 0; i < STAGES; ++i) issue();

  int taken = 0;
  bool good = true;
  for (long long seg = lo; seg < hi;) {
    // a tile of rows, or the part of it that is this block's: records first .. last - 1 of the tile
    const int first = here.i, last = (int)min((long long)here.each, first + (hi - seg));
    const int rows = min(ROWS, here.q.rows.n * p.group - here.tile * ROWS), base = here.q.rows.len - here.q.rows.n;
    int pos[NT][2];                                        // of the columns of S^T that the lane holds
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int b = 0; b < 2; ++b) pos[n][b] = base + min(here.tile * ROWS + 8 * n + 2 * t + b, here.q.rows.n * p.group - 1) / p.group;
    if constexpr (Smem::Q_HERE) {
      if (warp == 0) load_q(here);
      __syncthreads();
    }
    const int first_at = base + here.tile * ROWS / p.group, last_at = base + (here.tile * ROWS + rows - 1) / p.group;
    float o[NK][NT][4] = {};
    float top[NT][2], move[NT][2] = {}, sum[NT][2] = {};   // top: the rows' references; sum: of the lane's tokens
    bool far = false;                                      // (some of the warp's rows' are)
#pragma unroll
    for (int n = 0; n < NT; ++n) top[n][0] = top[n][1] = -INFINITY;
    // the warp's records are every WARPS-th of the block's
    int i = first + (int)((warp + WARPS - (seg - lo) % WARPS) % WARPS);
    for (; i < last; i += WARPS) {
      const int st = taken % STAGES;
      if (good) good = mbar_wait_warp(smem_u32(&sm.bars[warp][st]), (taken / STAGES) & 1, &sm.abort_flag, p.status, LQ_STAGE_DRAIN);
      if (!good) break;
      ++taken;
      const uint8_t* rec = sm.ring[warp][st];
      const uint4* ku = reinterpret_cast<const uint4*>(rec + LQ_KV_HEAD) + lane;
      const uint4* vu = ku + 2 * DP;
      if (!sm.empty[warp][st]) {
        const uint32_t head = *reinterpret_cast<const uint32_t*>(rec);
        const int token0 = here.q.seen.block(i) * LQ_KV_BLOCK;
        float s[2][NT][4] = {};                            // [words 2 a, 2 a + 1][..][token of word 2 a: rows 2 t, 2 t + 1; of 2 a + 1]
        {
          const uint32_t high = lq_kv_high((int8_t)(head & 0xFF));
          const __half2 less = lq_kv_less(high);
#pragma unroll
          for (int g = 0; g < NK; ++g) {
            const uint4 w = ku[32 * g];
            const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int a = 0; a < 2; ++a) {
              const uint32_t a0 = lq_kv_open<0x4140>(ww[2 * a], high, less), a2 = lq_kv_open<0x4342>(ww[2 * a], high, less);
              const uint32_t a1 = lq_kv_open<0x4140>(ww[2 * a + 1], high, less), a3 = lq_kv_open<0x4342>(ww[2 * a + 1], high, less);
#pragma unroll
              for (int n = 0; n < NT; ++n) {
                if constexpr (Smem::Q_HERE) mma_f16(s[a][n], a0, a1, a2, a3, sm.q[g][n][lane]);
                else mma_f16(s[a][n], a0, a1, a2, a3, qb[g][n]);
              }
            }
          }
        }
        if (!lq_all_seen(p, first_at, last_at, token0, token0 + LQ_KV_BLOCK - 1, here.q.rows.len)) {
#pragma unroll
          for (int a = 0; a < 2; ++a)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int x = 0; x < 4; ++x)
                if (!lq_sees(p, pos[n][x & 1], token0 + lq_kv_token(c8, 2 * a + (x >> 1)), here.q.rows.len)) s[a][n][x] = -INFINITY;
        }
        float high_s[NT][2];
        bool grow = far;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            high_s[n][b] = fmaxf(fmaxf(s[0][n][b], s[0][n][2 + b]), fmaxf(s[1][n][b], s[1][n][2 + b]));
            grow = grow || (high_s[n][b] - top[n][b]) * scale > LQ_ATTN_GROWTH;
          }
        if (__any_sync(0xffffffffu, grow)) {
          bool out = false;
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              float m = high_s[n][b];
#pragma unroll
              for (int d = 4; d < 32; d *= 2) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
              m = fmaxf(m, top[n][b]);
              // (a row that has seen nothing yet has sums of zero)
              const float by = top[n][b] == -INFINITY ? 1.f : ex2((top[n][b] - m) * scale);
              top[n][b] = m;
              move[n][b] = lq_attn_move(m, scale);
              out = out || lq_attn_far(m, scale);
              sum[n][b] *= by;
#pragma unroll
              for (int g = 0; g < NK; ++g) { o[g][n][b] *= by; o[g][n][2 + b] *= by; }
            }
          far = __any_sync(0xffffffffu, out);
          if (far) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int b = 0; b < 2; ++b) {
                const float off = lq_attn_far(top[n][b], scale) ? top[n][b] : 0.f;
#pragma unroll
                for (int a = 0; a < 2; ++a) { s[a][n][b] -= off; s[a][n][2 + b] -= off; }
              }
          }
        }
        uint2 w[2][NT];                                    // weights of 16 tokens: of words 2 a, of words 2 a + 1
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          const float r0 = move[n][0], r1 = move[n][1];
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const float x0 = ex2(fmaf(s[a][n][0], scale, r0)), x1 = ex2(fmaf(s[a][n][1], scale, r1));
            const float x2 = ex2(fmaf(s[a][n][2], scale, r0)), x3 = ex2(fmaf(s[a][n][3], scale, r1));
            sum[n][0] += x0 + x2;
            sum[n][1] += x1 + x3;
            w[a][n] = make_uint2(turned(pack(x0, x1)), turned(pack(x2, x3)));
          }
        }
        const uint32_t high = lq_kv_high((int8_t)(head >> 8 & 0xFF));
        const __half2 less = lq_kv_less(high);
        // columns 2 t and 2 t + 1 of words 2 a are tokens 0 and 2 of the lane's four, of words 2 a + 1 tokens 1 and 3
#pragma unroll
        for (int g = 0; g < NK; ++g) {
          const uint4 v = vu[32 * g];
          const uint32_t vv[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
          for (int a = 0; a < 2; ++a) {
            const uint32_t a0 = lq_kv_open<0x4240>(vv[2 * a], high, less), a2 = lq_kv_open<0x4341>(vv[2 * a], high, less);
            const uint32_t a1 = lq_kv_open<0x4240>(vv[2 * a + 1], high, less), a3 = lq_kv_open<0x4341>(vv[2 * a + 1], high, less);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(o[g][n], a0, a1, a2, a3, w[a][n]);
          }
        }
      }
      fence_proxy_async();                                 // the stage is read by all lanes before a copy into it is asked for
      __syncwarp();
      issue();
    }
    const Place was = here;
    const long long next = seg + (last - first);
    if (next < hi) {
      if (!lq_attn_walk(here, last - first, p.b.heads, p.b.sequences, sequence)) break;
      if constexpr (!Smem::Q_HERE) load_q(here);
    }
    // the warps' results of the tile
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int b = 0; b < 2; ++b) {
#pragma unroll
        for (int d = 4; d < 32; d *= 2) sum[n][b] += __shfl_xor_sync(0xffffffffu, sum[n][b], d);
        const int row = 8 * n + 2 * t + b;
        if (row < rows) {
          if (c8 == 0) { sm.top[warp][row] = top[n][b]; sm.total[warp][row] = sum[n][b]; }
          if (top[n][b] != -INFINITY)
#pragma unroll
            for (int g = 0; g < NK; ++g) *reinterpret_cast<float2*>(&sm.sums[warp][row][16 * g + 2 * c8]) = make_float2(o[g][n][b], o[g][n][2 + b]);
        }
      }
    __syncthreads();
    const long long tile_begin = seg - first;
    const bool whole = first == 0 && last == was.each;
    const auto put = [&](int row, int d, float4 x, float total_w) {
      // values were opened as 2^-4 of themselves
      const float by = total_w > 0.f ? 16.f / total_w : 0.f;
      if (d >= p.D) return;
      const int r = was.tile * ROWS + row, tok = r / p.group;
      __half* to = p.out + (was.q.rows.row + tok) * p.out_row + (long long)(was.head * p.group + r - tok * p.group) * p.out_head + d;
      *reinterpret_cast<uint2*>(to) = make_uint2(pack(x.x * by, x.y * by), pack(x.z * by, x.w * by));
    };
    float* part = p.part + (2ll * blockIdx.x + (first == 0 ? 1 : 0)) * LQ_ATTN_ROWS * (DP + 4);
    for (int e = tid; e < rows * (DP / 4); e += THREADS) {
      const int row = e / (DP / 4), d = 4 * (e - row * (DP / 4));
      float m = -INFINITY, n = 0.f;
      float tops[WARPS];
#pragma unroll
      for (int i = 0; i < WARPS; ++i) m = fmaxf(m, tops[i] = sm.top[i][row]);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < WARPS; ++i) {
        if (tops[i] == -INFINITY) continue;
        const float k = ex2((tops[i] - m) * scale);
        const float4 v = *reinterpret_cast<const float4*>(&sm.sums[i][row][d]);
        n = fmaf(k, sm.total[i][row], n);
        x.x = fmaf(k, v.x, x.x); x.y = fmaf(k, v.y, x.y); x.z = fmaf(k, v.z, x.z); x.w = fmaf(k, v.w, x.w);
      }
      if (whole) {
        put(row, d, x, n);
      } else {
        float* to = part + row * (DP + 4);
        *reinterpret_cast<float4*>(to + 4 + d) = x;
        if (d == 0) *reinterpret_cast<float2*>(to) = make_float2(m, n);
      }
    }
    if (!whole) {
      int from = blockIdx.x - sm.part, parts = sm.parts;   // the blocks that have some of the tile
      if (!cut.parted) {
        from = (int)lq_quotient(tile_begin, cut.share);
        parts = (int)lq_quotient(tile_begin + was.each - 1, cut.share) - from + 1;
      }
      __syncthreads();                                     // (behind this the count's release covers what all threads have written)
      if (tid == 0) {
        sm.last = add_acq_rel(&p.count[from], 1) == parts - 1;
        if (sm.last) p.count[from] = 0;                    // (nobody else comes)
      }
      __syncthreads();
      if (sm.last) {
        for (int e = tid; e < rows * (DP / 4); e += THREADS) {
          const int row = e / (DP / 4), d = 4 * (e - row * (DP / 4));
          float m = -INFINITY, n = 0.f;
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          for (int c = 0; c < parts; c += 4) {             // four at a time are on their way
            float2 head[4];
            float4 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float* at = p.part + ((2ll * (from + min(c + i, parts - 1)) + (c + i == 0 ? 1 : 0)) * LQ_ATTN_ROWS + row) * (DP + 4);
              head[i] = __ldcg(reinterpret_cast<const float2*>(at));
              v[i] = __ldcg(reinterpret_cast<const float4*>(at + 4 + d));
              if (c + i >= parts) head[i].x = -INFINITY;
            }
            const float top = fmaxf(m, fmaxf(fmaxf(head[0].x, head[1].x), fmaxf(head[2].x, head[3].x)));
            const float by = m == -INFINITY ? 0.f : ex2((m - top) * scale);
            n *= by; x.x *= by; x.y *= by; x.z *= by; x.w *= by;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              if (head[i].x == -INFINITY) continue;
              const float k = ex2((head[i].x - top) * scale);
              n = fmaf(k, head[i].y, n);
              x.x = fmaf(k, v[i].x, x.x); x.y = fmaf(k, v[i].y, x.y); x.z = fmaf(k, v[i].z, x.z); x.w = fmaf(k, v[i].w, x.w);
            }
            m = top;
          }
          put(row, d, x, n);
        }
      }
    }
    __syncthreads();                                       // the warps' results are read
    seg = next;
  }
  // (only after a wait that gave up: what is in flight lands before the block leaves)
  if (!good)
    for (; taken < issued; ++taken) mbar_settle(smem_u32(&sm.bars[warp][taken % STAGES]), (taken / STAGES) & 1);
}

// Shared memory holds two to four records of every warp and the warps' sums.
template <int NK, int NT, int WARPS, int STAGES>
struct Form {
  static cudaError_t launch(const lq_kvcache* C, const LqAttnParams& p, cudaStream_t st) {
    return lq_launch(lq_attn_kernel<NK, NT, WARPS, STAGES>, C->sms, 32 * WARPS, sizeof(Shared<NK, NT, WARPS, STAGES>), st, p);
  }
  static bool room() {
    return lq_note_cuda(cudaFuncSetAttribute(lq_attn_kernel<NK, NT, WARPS, STAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)sizeof(Shared<NK, NT, WARPS, STAGES>))) == cudaSuccess;
  }
};
template <typename F>
auto with_form(int Dp, bool narrow, const F& f) {
  switch (Dp) {
    case 64: return narrow ? f(Form<4, 1, 8, 4>()) : f(Form<4, 2, 8, 4>());
    case 80: return narrow ? f(Form<5, 1, 8, 3>()) : f(Form<5, 2, 8, 3>());
    case 96: return narrow ? f(Form<6, 1, 8, 3>()) : f(Form<6, 2, 8, 2>());
    case 112: return narrow ? f(Form<7, 1, 8, 2>()) : f(Form<7, 2, 8, 2>());
    case 128: return narrow ? f(Form<8, 1, 8, 2>()) : f(Form<8, 2, 8, 2>());
    case 192: return narrow ? f(Form<12, 1, 4, 3>()) : f(Form<12, 2, 4, 3>());
    default: return narrow ? f(Form<16, 1, 4, 2>()) : f(Form<16, 2, 4, 2>());
  }
}

}  // namespace

lq_status lq_attn_prepare(const lq_kvcache* C) {
  for (bool narrow : {false, true})
    if (!with_form(C->Dp, narrow, [](auto form) { return form.room(); })) return LQ_ERR_CUDA;
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
  if ((s = status(lq_runs_collide(out))) != LQ_OK || (s = status(lq_runs_meet(out, q))) != LQ_OK || (s = status(lq_batch_meets(p.b, p.b.row_start, p.b.sequences + 1, out))) != LQ_OK) return s;
  LqDeviceGuard guard(C->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  p.records = lq_kv_layer(C, layer);
  p.q = (const __half*)a->q; p.out = (__half*)a->out;
  p.q_row = a->q_row; p.q_head = a->q_head; p.out_row = a->out_row; p.out_head = a->out_head;
  p.D = C->D; p.group = a->q_heads / C->heads;
  p.causal = a->causal; p.window = a->window; p.sinks = a->sinks;
  p.scale = a->scale * 16.f * 1.44269504088896341f;        // (keys are opened as 2^-4 of themselves)
  p.part = C->d_part; p.count = C->d_count;
  p.tile_part = C->d_tile_part; p.tile_meta = C->d_tile_meta;
  p.status = lq_device_status_ptr(C->device);
  // Which form a sequence's rows are the kernels tell by themselves where sequences have different numbers of them; a form that no sequence can be is
  // not launched.
  const bool tiles = C->Dp <= 128;
  const int few = lq_attn_few(p.b.sequences, C->heads, C->sms);
  const long long most = p.b.row_start ? (long long)p.b.rows * p.group : (long long)p.b.each * p.group, least = p.b.row_start ? 1 : most;
  if (!tiles || least <= few) {
    p.few = 1;
    p.many = tiles ? few + 1 : 0x7fffffff;
    // (tiles of eight rows where no sequence has more)
    const cudaError_t e = with_form(C->Dp, most <= 8, [&](auto form) { return form.launch(C, p, (cudaStream_t)stream); });
    if (lq_note_cuda(e) != cudaSuccess) return LQ_ERR_CUDA;
  }
  if (tiles && most > few) {
    p.few = few + 1;
    p.many = 0x7fffffff;
    return lq_attn_tile_launch(C, p, (cudaStream_t)stream);
  }
  return LQ_OK;
}
