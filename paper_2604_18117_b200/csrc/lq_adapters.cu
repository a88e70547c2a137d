// Low-rank adapters of many requests beside a shared projection:  Y[m] = Y0[m] + scale_a (X[m] A_a) B_a,  a = the adapter of row m.
//
// A map sorts the rows of a batch by adapter (stable) and cuts them into tiles of rows of one adapter; every projection of a step
// uses it.  This file has the map, the set of adapters, and the forward for few rows; lq_adapters_tile.cu has the one for many.
//
// T = X A is summed in fp32 and enters the second product as two halves, hi + lo, under a power of two of its row: 22 bits of the row's
// largest entry, at the price of a second MMA for each 16 of the rank, which no form is bound by.  (One half would round T to 11 bits, as
// much as an fp16 output is rounded, and too much for an fp32 one.)
#include <math.h>

#include <algorithm>
#include <new>

#include "lq_adapters.h"
#include "lq_device.cuh"

using namespace lqdev;

namespace {

constexpr int MAX_SLOTS = 1023;      // bins of the sort: the slots and "none"
constexpr int WARPS = 8;
// most rows that one block sorts; more: eight blocks (us: 2048 rows 4.2 / 5.5, 8192 rows 6.6 / 5.7, 32768 rows 18.4 / 7.1)
constexpr int ROWMAP_SINGLE = 4096;

// ---- the map: a stable counting sort by one block, or by a cluster of them -----------------------------------------------
// Each warp counts the adapters of its own run of rows, then places them behind those of the warps before it.  What this costs is latency:
// up to eight loads of a warp are in flight together, a run of up to 256 rows is read once, and many rows are shared by eight blocks.  (64
// registers are all that 1024 threads can have; the form of eight blocks spills 52 bytes.)
template <int BLOCKS>
__global__ void __launch_bounds__(1024) lq_rowmap_kernel(const int32_t* ids, int M, int slots, int* perm, LqAdTile* tiles, LqAdTile* small,
                                                         int* ntiles) {
  extern __shared__ int count[];     // [32][slots + 1]
  __shared__ int scan_rows[32], scan_tiles[32], total[MAX_SLOTS + 1];
  constexpr int AHEAD = 8;
  const int bins = slots + 1, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, block = BLOCKS > 1 ? blockIdx.x : 0;
  const int run = ((M + 32 * BLOCKS - 1) / (32 * BLOCKS) + 31) & ~31;    // rows a warp: whole loads
  const long long first = (long long)(block * 32 + warp) * run;
  const int n = (int)max(0ll, min((long long)run, M - first)); // this warp's rows
  const int warps = (int)max(0ll, min(32ll, (M - (long long)block * 32 * run + run - 1) / run));     // of this block that have any
  for (int i = tid; i < warps * bins; i += 1024) count[i] = 0;
  grid_launch_dependents();
  grid_dependency_wait();
  int* mine = count + warp * bins;
  int bin[AHEAD];                                              // of the rows in hand; -1: no row
  const auto read = [&](int r0) {
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      const int r = r0 + 32 * u + lane;
      bin[u] = r < n ? ids[first + r] : -2;
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) bin[u] = r0 + 32 * u + lane < n ? (bin[u] >= 0 && bin[u] < slots ? bin[u] : slots) : -1;
  };
  read(0);
  __syncthreads();
  for (int r0 = 0; r0 < n; r0 += 32 * AHEAD) {
    if (r0 > 0) read(r0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (r0 + 32 * u >= n) break;
      const unsigned same = __match_any_sync(0xffffffffu, bin[u]);
      if (bin[u] >= 0 && lane == __ffs(same) - 1) mine[bin[u]] += __popc(same);
      __syncwarp();
    }
  }
  __syncthreads();
  // thread b: rows and tiles of bin b, and where they begin.  Tiles of 128 rows count from bit 12 on, tiles of 16, of which there are fewer
  // than 4096, below it
  int rows = 0, before = 0;
  if (tid < bins)
#pragma unroll
    for (int w = 0; w < 32; ++w) rows += w < warps ? count[w * bins + tid] : 0;
  if constexpr (BLOCKS > 1) {
    if (tid < bins) total[tid] = rows;
    cluster_sync();
    rows = 0;
    if (tid < bins) {
      int u[BLOCKS];
#pragma unroll
      for (int c = 0; c < BLOCKS; ++c)
        asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(u[c]) : "r"(peer_smem(smem_u32(total + tid), c)) : "memory");
#pragma unroll
      for (int c = 0; c < BLOCKS; ++c) {
        before += c < block ? u[c] : 0;
        rows += u[c];
      }
    }
  }
  const int large = (rows + LQ_AD_TILE - 1) / LQ_AD_TILE, little = M <= LQ_AD_SMALL_M ? (rows + LQ_AD_SMALL_TILE - 1) / LQ_AD_SMALL_TILE : 0;
  const int nt = large << 12 | little;
  int a = rows, b = nt;
#pragma unroll
  for (int d = 1; d < 32; d *= 2) {
    const int u = __shfl_up_sync(0xffffffffu, a, d), v = __shfl_up_sync(0xffffffffu, b, d);
    if (lane >= d) { a += u; b += v; }
  }
  if (lane == 31) { scan_rows[warp] = a; scan_tiles[warp] = b; }
  __syncthreads();
  if (warp == 0) {
    int u = scan_rows[lane], v = scan_tiles[lane];
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int x = __shfl_up_sync(0xffffffffu, u, d), y = __shfl_up_sync(0xffffffffu, v, d);
      if (lane >= d) { u += x; v += y; }
    }
    scan_rows[lane] = u; scan_tiles[lane] = v;
  }
  __syncthreads();
  if (tid == 0 && block == 0) *reinterpret_cast<int4*>(ntiles) = make_int4(scan_tiles[31] >> 12, scan_tiles[31] & 0xFFF, M, 0);
  if (tid < bins) {
    const int at0 = a - rows + (warp > 0 ? scan_rows[warp - 1] : 0);
    const int tile0 = b - nt + (warp > 0 ? scan_tiles[warp - 1] : 0), adapter = tid < slots ? tid : -1;
    for (int i = block; i < large; i += BLOCKS)
      tiles[(tile0 >> 12) + i] = LqAdTile{adapter, at0 + i * LQ_AD_TILE, min(LQ_AD_TILE, rows - i * LQ_AD_TILE), -1};
    for (int i = block; i < little; i += BLOCKS)
      small[(tile0 & 0xFFF) + i] = LqAdTile{adapter, at0 + i * LQ_AD_SMALL_TILE, min(LQ_AD_SMALL_TILE, rows - i * LQ_AD_SMALL_TILE), -1};
    int c[32], at = at0 + before;
#pragma unroll
    for (int w = 0; w < 32; ++w) c[w] = w < warps ? count[w * bins + tid] : 0;
#pragma unroll
    for (int w = 0; w < 32; ++w) {
      if (w < warps) count[w * bins + tid] = at;
      at += c[w];
    }
  }
  __syncthreads();
  for (int r0 = 0; r0 < n; r0 += 32 * AHEAD) {
    if (run > 32 * AHEAD) read(r0);
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
      if (r0 + 32 * u >= n) break;
      const unsigned same = __match_any_sync(0xffffffffu, bin[u]);
      const int at = bin[u] >= 0 ? mine[bin[u]] + __popc(same & ((1u << lane) - 1)) : 0;
      __syncwarp();
      if (bin[u] >= 0) {
        perm[at] = (int)first + r0 + 32 * u + lane;
        if (lane == __ffs(same) - 1) mine[bin[u]] += __popc(same);
      }
      __syncwarp();
    }
  }
  // large tiles whose rows are neighbours (perm ascends within a tile)
  if constexpr (BLOCKS > 1) {
    cluster_sync();                                            // (and the others have read this block's totals)
  } else {
    if (M <= LQ_AD_ANY_M) return;
    __syncthreads();
  }
  for (int i = block * 1024 + tid; i < scan_tiles[31] >> 12; i += 1024 * BLOCKS) {
    const LqAdTile t = tiles[i];
    const int r = perm[t.begin];
    if (perm[t.begin + t.rows - 1] - r == t.rows - 1) tiles[i].first = r;
  }
}

// ---- a slot's new adapter in the forwards' layouts ----------------------------------------------------------------------
__global__ void __launch_bounds__(256) lq_adapters_set_kernel(__half* down, __half* up, LqAdMeta* meta, const __half* A, const __half* B, int K,
                                                              int N, int Npad, int rp, int rank, float scale) {
  grid_dependency_wait();            // (no launch_dependents: what follows sees the adapter whole)
  const long long n_down = (long long)rp * K, n_up = (long long)Npad * rp, step = (long long)gridDim.x * blockDim.x;
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < n_down + n_up; i += step) {
    if (i < n_down) {
      const int j = (int)(i / K), k = (int)(i - (long long)j * K);
      down[i] = j < rank ? A[(long long)k * rank + j] : __half(0.f);
    } else {
      const long long e = i - n_down;
      const int s = (int)(e / rp), j = (int)(e - (long long)s * rp);
      const int n = (s & ~31) | (((s >> 3) & 3) << 1) | (((s >> 1) & 3) << 3) | (s & 1);      // the column whose slot is s: the map is its own inverse
      up[e] = j < rank && n < N ? B[(long long)j * N + n] : __half(0.f);
    }
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *meta = LqAdMeta{rank, scale};
}

// ---- fragments ---------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void mma_16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// L1: a copy takes half of a 32-byte sector and another one the rest (1365 rows, 1160 x 2312, fp32: 20.7 us, without 22.7)
template <int BYTES, bool L1 = false>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src) {
  if constexpr (BYTES == 16 && L1) asm volatile("cp.async.ca.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// bytes of a warp's places for what is fetched ahead
__host__ __device__ constexpr int adapters_stage(int rp, bool f32) { return ((rp <= 32 ? 4 : 0) + (f32 ? 4 : 2)) * 512; }

// The forward for few rows: a cluster of CTAs has 16 rows of one adapter, shares out K for the first product, joins the sums through
// distributed shared memory (each CTA all of them, always in the same order) and shares out the columns for the second.  A chain of
// latencies: one launch, and operands straight from global memory into the fragments of mma.sync (tiles of 16 rows would leave tcgen05's 128
// empty).  The order of a product's inner index is free as long as both operands have the same: lane (g, t) takes the eight neighbours 8 t ..
// 8 t + 7 of each 32, so that a fragment of either operand is one 16-byte load from rows that run along the inner index.  us with the map:
// one row, 1152 x 1152, rank 16 7.3; 64 rows with an adapter each, 1152 x 4608, rank 32 15.0 (25 MB of factors: 3.8 at the measured copy
// rate); of these 3.4 are the map.  The first columns' B and Y0 are on their way during the first product, through shared memory (asked for
// where they are used 15.3; ahead through registers, which spill, 22.7).
template <int RP, int CLUSTER, bool F32>
__global__ void __launch_bounds__(32 * WARPS, RP <= 32 ? 4 : 3)
    lq_adapters_kernel(const LqAdTile* tiles, const int* ntiles, int M, int32_t* status, const int* perm, const __half* X, const void* Y0, void* Y,
                       const __half* down, const __half* up, const LqAdMeta* meta, int K, int N, int Npad) {
  constexpr int NT = RP / 8, KB = (RP + 31) / 32;
  extern __shared__ __align__(16) float smem[];
  float* red = smem;                                      // [WARPS][16][RP]
  float* part = red + WARPS * 16 * RP;                    // [16][RP] this CTA's share of K
  __half* tq = reinterpret_cast<__half*>(part + 16 * RP); // [2][16][KB * 32]: hi, lo
  float* row_scale = reinterpret_cast<float*>(tq + 2 * 16 * KB * 32);   // [16]
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int rank_in_cluster = blockIdx.x % CLUSTER, ti = blockIdx.x / CLUSTER;
  grid_launch_dependents();
  grid_dependency_wait();
  // (a tile behind the last one holds anything: it is asked for together with their number, which saves a trip)
  const LqAdTile tile = tiles[ti];
  if (ti >= lq_ad_tiles_of<true>(ntiles, M, status)) return;            // (the whole cluster)
  const LqAdMeta m = tile.adapter >= 0 ? meta[tile.adapter] : LqAdMeta{0, 0.f};
  const int unit = warp * CLUSTER + rank_in_cluster, units = WARPS * CLUSTER;
  const bool has0 = g < tile.rows, has1 = g + 8 < tile.rows;
  const long long row0 = has0 ? perm[tile.begin + g] : 0, row1 = has1 ? perm[tile.begin + g + 8] : 0;
  if (m.rank == 0 && Y == Y0) return;
  // What the lane adds to and, of narrow factors, its B, for the first columns and then for the next ones, without registers: through places
  // of shared memory that no other lane looks at.
  constexpr int YW = F32 ? 2 : 1;                         // 16-byte words of eight columns
  constexpr bool STAGE_B = RP <= 32;
  const uint32_t stage = smem_u32(row_scale + 16) + warp * adapters_stage(RP, F32) + lane * 16;
  const __half* Bu = up + (long long)max(tile.adapter, 0) * Npad * RP;
  const auto fetch = [&](int cg) {
    if (cg * 32 >= N) return;
    if (STAGE_B && m.rank > 0)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const __half* src = Bu + (long long)(32 * cg + 8 * j + g) * RP;
        if constexpr (RP == 16) cp_async<8>(stage + (2 * YW + j) * 512, src + 4 * t);        // half a block: four neighbours a lane
        else cp_async<16>(stage + (2 * YW + j) * 512, src + 8 * t);
      }
    const int n = 32 * cg + 8 * t;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (n < N && (h ? has1 : has0)) {
        const unsigned char* src = reinterpret_cast<const unsigned char*>(Y0) + ((h ? row1 : row0) * N + n) * (F32 ? 4 : 2);
#pragma unroll
        for (int w = 0; w < YW; ++w) cp_async<16, F32>(stage + (YW * h + w) * 512, src + 16 * w);
      }
  };
  fetch(unit);

  float c[NT][4];
  if (m.rank > 0) {
#pragma unroll
    for (int n = 0; n < NT; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
    const __half* A = down + (long long)tile.adapter * RP * K;
    for (int kb = unit; kb * 32 < K; kb += units) {
      const int k = kb * 32 + 8 * t;
      const uint4 zero = make_uint4(0, 0, 0, 0);
      const bool in = k < K;
      const uint4 x0 = in && has0 ? *reinterpret_cast<const uint4*>(X + row0 * K + k) : zero;
      const uint4 x1 = in && has1 ? *reinterpret_cast<const uint4*>(X + row1 * K + k) : zero;
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (n * 8 < m.rank) {
          const uint4 b = in ? *reinterpret_cast<const uint4*>(A + (long long)(8 * n + g) * K + k) : zero;
          mma_16816(c[n], x0.x, x1.x, x0.y, x1.y, b.x, b.y);
          mma_16816(c[n], x0.z, x1.z, x0.w, x1.w, b.z, b.w);
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      *reinterpret_cast<float2*>(red + (warp * 16 + g) * RP + 8 * n + 2 * t) = make_float2(c[n][0], c[n][1]);
      *reinterpret_cast<float2*>(red + (warp * 16 + g + 8) * RP + 8 * n + 2 * t) = make_float2(c[n][2], c[n][3]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 16 * RP; i += 32 * WARPS) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) s += red[w * 16 * RP + i];
      part[i] = s;
    }
    cluster_sync();
    // every CTA adds up the whole intermediate, always in the same order, two rows a warp
    for (int r = 2 * warp; r < 2 * warp + 2; ++r) {
      float v[KB];
      float top = 0.f;
#pragma unroll
      for (int q = 0; q < KB; ++q) {
        const int j = 32 * q + lane;
        v[q] = 0.f;
        if (j < RP)
#pragma unroll
          for (int w = 0; w < CLUSTER; ++w) {
            float u;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u) : "r"(peer_smem(smem_u32(part + r * RP + j), w)) : "memory");
            v[q] += u;
          }
        top = fmaxf(top, fabsf(v[q]));
      }
#pragma unroll
      for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      const int e = lq_ad_exponent(top);
      if (lane == 0) row_scale[r] = ldexpf(m.scale, -e);
#pragma unroll
      for (int q = 0; q < KB; ++q) {
        const float u = ldexpf(v[q], e);
        const __half hi = __float2half_rn(u);
        tq[r * KB * 32 + 32 * q + lane] = hi;
        tq[(16 + r) * KB * 32 + 32 * q + lane] = __float2half_rn(u - __half2float(hi));
      }
    }
    cluster_arrive<false>();                              // this CTA has read the others' shares
    __syncthreads();
  }
  const float s0 = m.rank > 0 ? row_scale[g] : 0.f, s1 = m.rank > 0 ? row_scale[g + 8] : 0.f;
  for (int cg = unit; cg * 32 < N; cg += units) {
    float d[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) d[j][0] = d[j][1] = d[j][2] = d[j][3] = 0.f;
    const int n = 32 * cg + 8 * t;                        // this lane's eight columns
    cp_async_wait();
    if (m.rank > 0) {
#pragma unroll
      for (int q = 0; q < KB; ++q)
        if (32 * q < m.rank) {
          uint4 b[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            if constexpr (STAGE_B) b[j] = lds_v4(stage + (2 * YW + j) * 512);
            else b[j] = *reinterpret_cast<const uint4*>(Bu + (long long)(32 * cg + 8 * j + g) * RP + 32 * q + 8 * t);
          }
#pragma unroll
          for (int part_of = 0; part_of < 2; ++part_of) {
            const __half* a0p = tq + (16 * part_of + g) * KB * 32 + 32 * q + (RP == 16 ? 4 : 8) * t;
            const __half* a1p = a0p + 8 * KB * 32;
            if constexpr (RP == 16) {
              const uint2 a0 = *reinterpret_cast<const uint2*>(a0p), a1 = *reinterpret_cast<const uint2*>(a1p);
#pragma unroll
              for (int j = 0; j < 4; ++j) mma_16816(d[j], a0.x, a1.x, a0.y, a1.y, b[j].x, b[j].y);
            } else {
              const uint4 a0 = *reinterpret_cast<const uint4*>(a0p), a1 = *reinterpret_cast<const uint4*>(a1p);
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                mma_16816(d[j], a0.x, a1.x, a0.y, a1.y, b[j].x, b[j].y);
                mma_16816(d[j], a0.z, a1.z, a0.w, a1.w, b[j].z, b[j].w);
              }
            }
          }
        }
    }
    uint4 y[2][YW];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const float s = h ? s1 : s0;
#pragma unroll
      for (int w = 0; w < YW; ++w) y[h][w] = lds_v4(stage + (YW * h + w) * 512);
      if (m.rank > 0) {                                   // (a row without an adapter keeps its bits)
        if constexpr (F32) {
          float* f = reinterpret_cast<float*>(&y[h][0]);
#pragma unroll
          for (int j = 0; j < 8; ++j) f[j] = fmaf(s, d[j / 2][2 * h + j % 2], f[j]);
        } else {
          __half2* w = reinterpret_cast<__half2*>(&y[h][0]);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float2 f = __half22float2(w[j]);
            w[j] = __floats2half2_rn(fmaf(s, d[j][2 * h], f.x), fmaf(s, d[j][2 * h + 1], f.y));
          }
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if (n < N && (h ? has1 : has0)) {
        uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<unsigned char*>(Y) + ((h ? row1 : row0) * N + n) * (F32 ? 4 : 2));
#pragma unroll
        for (int w = 0; w < YW; ++w) to[w] = y[h][w];
      }
    fetch(cg + units);                                    // (behind the stores: what is here has been read by then)
  }
  if (m.rank > 0) cluster_wait();                         // the others have read this CTA's share
}

size_t forward_smem(int rp, bool f32) {
  const int kb = (rp + 31) / 32;
  return (size_t)(WARPS + 1) * 16 * rp * 4 + 2 * 16 * kb * 32 * 2 + 16 * 4 + (size_t)WARPS * adapters_stage(rp, f32);
}
template <int RP, int CLUSTER>
cudaError_t launch_cluster(const lq_adapters* S, const lq_rowmap* R, int tiles, const void* X, const void* Y0, void* Y, lq_out_dtype dt, cudaStream_t st) {
  const bool f32 = dt == LQ_OUT_F32;
  return lq_launch_cluster(f32 ? lq_adapters_kernel<RP, CLUSTER, true> : lq_adapters_kernel<RP, CLUSTER, false>, tiles * CLUSTER, 32 * WARPS, CLUSTER,
                           forward_smem(RP, f32), st, (const LqAdTile*)R->d_small, (const int*)R->d_ntiles, R->M, lq_device_status_ptr(R->device),
                           (const int*)R->d_perm, (const __half*)X, Y0, Y, (const __half*)S->d_down, (const __half*)S->d_up, (const LqAdMeta*)S->d_meta,
                           S->K, S->N, S->Npad);
}
template <int RP>
cudaError_t launch_forward(const lq_adapters* S, const lq_rowmap* R, const void* X, const void* Y0, void* Y, lq_out_dtype dt, cudaStream_t st) {
  // Eight CTAs a tile while all of them are resident at once, else four (us with the map, eight / four: 1400 rows, 1152 x 3456, rank 32 25.8
  // / 20.9; 64 rows with an adapter each, 512 x 8192, rank 64 43.4 / 32.3; one row, 1152 x 3456, rank 32 9.2 / 11.2; two were never better).
  const int tiles = lq_ad_tiles(R->M, R->slots, LQ_AD_SMALL_TILE), resident = (RP <= 32 ? 4 : 3) * R->sms;
  return 8 * tiles <= resident ? launch_cluster<RP, 8>(S, R, tiles, X, Y0, Y, dt, st) : launch_cluster<RP, 4>(S, R, tiles, X, Y0, Y, dt, st);
}
template <int RP, typename Room>
bool room_of_rank(const Room& room) {
  return room(lq_adapters_kernel<RP, 8, false>, forward_smem(RP, false)) && room(lq_adapters_kernel<RP, 8, true>, forward_smem(RP, true)) &&
         room(lq_adapters_kernel<RP, 4, false>, forward_smem(RP, false)) && room(lq_adapters_kernel<RP, 4, true>, forward_smem(RP, true));
}

}  // namespace

extern "C" lq_status lq_adapters_create(int32_t K, int32_t N, int32_t max_rank, int32_t slots, int device, lq_adapters** out) {
  if (!out || K <= 0 || N <= 0 || max_rank <= 0 || slots <= 0) return LQ_ERR_INVALID_ARG;
  if (K > LQ_MAX_K || K % 8 != 0 || N % 8 != 0 || N > (1 << 20) || max_rank > LQ_MAX_RANK || slots > MAX_SLOTS) return LQ_ERR_UNSUPPORTED;
  int ndev = 0;
  if (lq_note_cuda(cudaGetDeviceCount(&ndev)) != cudaSuccess || device < 0 || device >= ndev) return LQ_ERR_CUDA;
  LqDeviceGuard guard(device);
  if (!guard.ok) return LQ_ERR_CUDA;
  lq_adapters* S = new (std::nothrow) lq_adapters();
  if (!S) return LQ_ERR_ALLOC;
  S->K = K; S->N = N; S->Npad = lq_round_up(N, 32); S->max_rank = max_rank; S->slots = slots; S->device = device;
  S->rp = max_rank <= 16 ? 16 : lq_round_up(max_rank, 32);
  const size_t n_down = (size_t)slots * S->rp * K, n_up = (size_t)slots * S->Npad * S->rp;
  if (lq_note_cuda(cudaMalloc((void**)&S->d_down, n_down * 2)) != cudaSuccess || lq_note_cuda(cudaMalloc((void**)&S->d_up, n_up * 2)) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&S->d_meta, slots * sizeof(LqAdMeta))) != cudaSuccess) {
    lq_adapters_free(S);
    return LQ_ERR_ALLOC;
  }
  // (what the factors of an empty slot hold reaches no output)
  if (lq_note_cuda(cudaMemset(S->d_meta, 0, slots * sizeof(LqAdMeta))) != cudaSuccess || lq_note_cuda(cudaDeviceSynchronize()) != cudaSuccess) {
    lq_adapters_free(S);
    return LQ_ERR_CUDA;
  }
  lq_status s;
  if ((s = lq_make_tmap_bytes(&S->tmDown, S->d_down, (uint64_t)slots * S->rp, (uint64_t)K * 2, (uint32_t)S->rp)) != LQ_OK ||
      (s = lq_make_tmap_bytes(&S->tmUp, S->d_up, (uint64_t)slots * S->Npad, (uint64_t)S->rp * 2, LQ_AD_TILE)) != LQ_OK) {
    lq_adapters_free(S);
    return s;
  }
  *out = S;
  return LQ_OK;
}

extern "C" lq_status lq_adapters_free(lq_adapters* S) {
  if (!S) return LQ_ERR_INVALID_ARG;
  LqDeviceGuard guard(S->device);
  cudaFree(S->d_down); cudaFree(S->d_up); cudaFree(S->d_meta);
  delete S;
  return LQ_OK;
}

extern "C" lq_status lq_adapters_set(lq_adapters* S, int32_t slot, int32_t rank, const void* A, const void* B, float scale, void* stream) {
  if (!S || slot < 0 || slot >= S->slots || rank < 0) return LQ_ERR_INVALID_ARG;
  if (rank > S->max_rank) return LQ_ERR_UNSUPPORTED;
  if (rank > 0 && (!A || !B || (((uintptr_t)A | (uintptr_t)B) & 1) != 0)) return LQ_ERR_INVALID_ARG;
  if (!isfinite(scale)) return LQ_ERR_NUMERIC;
  // A row's sums are below 2^46 (8192 products of halves), so their power of two is 2^-31 at least and scale / that a float; a larger scale
  // would be an infinity, and nothing times it no number.
  if (rank > 0 && fabsf(scale) >= 0x1p96f) return LQ_ERR_UNSUPPORTED;
  LqDeviceGuard guard(S->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  if (rank == 0)                     // nothing to lay out
    return lq_note_cuda(cudaMemsetAsync(S->d_meta + slot, 0, sizeof(LqAdMeta), (cudaStream_t)stream)) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
  const int blocks = (int)std::min(((long long)S->rp * (S->K + S->Npad) + 255) / 256, 4096ll);
  const size_t at = (size_t)slot * S->rp;
  const cudaError_t e = lq_launch(lq_adapters_set_kernel, blocks, 256, 0, (cudaStream_t)stream, S->d_down + at * S->K, S->d_up + at * S->Npad,
                                  S->d_meta + slot, (const __half*)A, (const __half*)B, S->K, S->N, S->Npad, S->rp, rank, scale);
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}

extern "C" lq_status lq_rowmap_create(int32_t M_max, int32_t slots, int device, lq_rowmap** out) {
  if (!out || M_max <= 0 || slots <= 0) return LQ_ERR_INVALID_ARG;
  if (slots > MAX_SLOTS || M_max > (1 << 24)) return LQ_ERR_UNSUPPORTED;
  int ndev = 0;
  if (lq_note_cuda(cudaGetDeviceCount(&ndev)) != cudaSuccess || device < 0 || device >= ndev) return LQ_ERR_CUDA;
  LqDeviceGuard guard(device);
  if (!guard.ok) return LQ_ERR_CUDA;
  lq_rowmap* R = new (std::nothrow) lq_rowmap();
  if (!R) return LQ_ERR_ALLOC;
  R->M_max = M_max; R->slots = slots; R->device = device; R->M = 0;
  const size_t rows = (size_t)M_max + LQ_AD_TILE;
  const size_t large = (size_t)lq_ceil_div(M_max, LQ_AD_TILE) + slots + 1;
  const size_t little = (size_t)lq_ceil_div(std::min(M_max, LQ_AD_SMALL_M), LQ_AD_SMALL_TILE) + slots + 1;
  if (lq_note_cuda(cudaDeviceGetAttribute(&R->sms, cudaDevAttrMultiProcessorCount, device)) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&R->d_ntiles, sizeof(int4))) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&R->d_tiles, large * sizeof(LqAdTile))) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&R->d_small, little * sizeof(LqAdTile))) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&R->d_perm, (size_t)M_max * sizeof(int))) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&R->d_T, rows * LQ_AD_TROW * 2)) != cudaSuccess ||
      lq_note_cuda(cudaMalloc((void**)&R->d_rscale, rows * sizeof(float))) != cudaSuccess) {
    lq_rowmap_free(R);
    return LQ_ERR_ALLOC;
  }
  // (no rows yet; T's rows are read in whole tiles: from defined contents on)
  lq_status s;
  if (lq_note_cuda(cudaMemset(R->d_ntiles, 0, sizeof(int4))) != cudaSuccess || lq_note_cuda(cudaMemset(R->d_T, 0, rows * LQ_AD_TROW * 2)) != cudaSuccess ||
      lq_note_cuda(cudaDeviceSynchronize()) != cudaSuccess) {
    lq_rowmap_free(R);
    return LQ_ERR_CUDA;
  }
  if (!lq_device_status_ptr(device)) {                      // (allocated here, not under a capture)
    lq_rowmap_free(R);
    return LQ_ERR_CUDA;
  }
  if ((s = lq_make_tmap_bytes(&R->tmT, R->d_T, rows, LQ_AD_TROW * 2, LQ_AD_TILE)) != LQ_OK || (s = lq_adapters_tiles_prepare()) != LQ_OK) {
    lq_rowmap_free(R);
    return s;
  }
  const auto room = [](auto* kernel, size_t bytes) {
    return lq_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes)) == cudaSuccess;
  };
  if (!room(lq_rowmap_kernel<1>, 32 * (MAX_SLOTS + 1) * 4) || !room(lq_rowmap_kernel<8>, 32 * (MAX_SLOTS + 1) * 4) || !room_of_rank<16>(room) ||
      !room_of_rank<32>(room) || !room_of_rank<64>(room)) {
    lq_rowmap_free(R);
    return LQ_ERR_CUDA;
  }
  *out = R;
  return LQ_OK;
}

extern "C" lq_status lq_rowmap_free(lq_rowmap* R) {
  if (!R) return LQ_ERR_INVALID_ARG;
  LqDeviceGuard guard(R->device);
  cudaFree(R->d_ntiles); cudaFree(R->d_tiles); cudaFree(R->d_small); cudaFree(R->d_perm); cudaFree(R->d_T); cudaFree(R->d_rscale);
  delete R;
  return LQ_OK;
}

extern "C" lq_status lq_rowmap_set(lq_rowmap* R, const int32_t* ids, int32_t M, void* stream) {
  if (!R || !ids || M <= 0 || M > R->M_max || ((uintptr_t)ids & 3) != 0) return LQ_ERR_INVALID_ARG;
  LqDeviceGuard guard(R->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  const size_t smem = (size_t)32 * (R->slots + 1) * 4;
  const auto launch = [&](auto* kernel, int blocks) {
    return lq_launch_cluster(kernel, blocks, 1024, blocks, smem, (cudaStream_t)stream, ids, M, R->slots, R->d_perm, R->d_tiles, R->d_small, R->d_ntiles);
  };
  const cudaError_t e = M > ROWMAP_SINGLE ? launch(lq_rowmap_kernel<8>, 8) : launch(lq_rowmap_kernel<1>, 1);
  if (lq_note_cuda(e) != cudaSuccess) return LQ_ERR_CUDA;
  R->M = M;
  return LQ_OK;
}

extern "C" lq_status lq_adapters_forward(const lq_adapters* S, const lq_rowmap* R, const void* X, const void* Y0, void* Y, lq_out_dtype dt, void* stream) {
  if (!S || !R || !X || !Y0 || !Y) return LQ_ERR_INVALID_ARG;
  if (S->device != R->device || R->slots > S->slots || R->M <= 0) return LQ_ERR_INVALID_ARG;
  if (dt != LQ_OUT_F16 && dt != LQ_OUT_F32) return LQ_ERR_INVALID_ARG;
  if ((((uintptr_t)X | (uintptr_t)Y0 | (uintptr_t)Y) & 15) != 0) return LQ_ERR_INVALID_ARG;
  const size_t y_bytes = (size_t)R->M * S->N * (dt == LQ_OUT_F32 ? 4 : 2);
  if ((Y0 != Y && lq_overlap(Y0, y_bytes, Y, y_bytes)) || lq_overlap(X, (size_t)R->M * S->K * 2, Y, y_bytes)) return LQ_ERR_INVALID_ARG;
  LqDeviceGuard guard(S->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  cudaStream_t st = (cudaStream_t)stream;
  if (!lq_ad_small_form(R->M, S->rp)) return lq_adapters_forward_tiles(S, R, X, Y0, Y, dt, st);
  const cudaError_t e = S->rp == 16   ? launch_forward<16>(S, R, X, Y0, Y, dt, st)
                        : S->rp == 32 ? launch_forward<32>(S, R, X, Y0, Y, dt, st)
                                      : launch_forward<64>(S, R, X, Y0, Y, dt, st);
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
