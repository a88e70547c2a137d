// Low-rank adapters, the form for many rows: two kernels on tiles of 128 rows of one adapter.
//
//   down   T = X A of a tile, K shared by a cluster of CTAs; each row of T leaves as two halves under a power of two
//   up     Y = Y0 + (scale / power of two) T B, tile by tile and 128 columns at a time
//
// X is read once, Y0 once, Y is written once; T is 512 bytes a row at most and stays in the L2, the factors too.  Once under way the up kernel
// runs at the memory's rate and the down kernel at 4 to 5 TB/s; of 8192 rows (13 to 31 us each, the memory busy 18 to 44 % of it) each spends 4 to
// 5 us in starting and ending.
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "lq_adapters.h"
#include "lq_device.cuh"

using namespace lqdev;

namespace {

constexpr int BM = LQ_AD_TILE, A_STAGE = BM * 128;      // a stage: 64 halves of K
constexpr int MAX_STAGES = 8;

// four rows of a tensor, wherever they lie
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* tm, int x, const int4& rows, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];" ::"r"(dst),
               "l"(reinterpret_cast<uint64_t>(tm)), "r"(x), "r"(rows.x), "r"(rows.y), "r"(rows.z), "r"(rows.w), "r"(bar)
               : "memory");
}
// the four rows that a lane fetches of a tile (behind the tile's last row: that one again)
__device__ __forceinline__ int4 tile_rows4(const int* perm, int rows, int lane) {
  return make_int4(perm[min(4 * lane, rows - 1)], perm[min(4 * lane + 1, rows - 1)], perm[min(4 * lane + 2, rows - 1)], perm[min(4 * lane + 3, rows - 1)]);
}
__device__ __forceinline__ float4 ld_peer_v4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_release(int* p, int v) { asm volatile("st.release.gpu.global.s32 [%0], %1;" ::"l"(p), "r"(v) : "memory"); }
__device__ __forceinline__ int ld_acquire(const int* p) {
  int v;
  asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t pack_halves(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Copies 128 bytes at x of each of a tile's rows.  Neighbours: in one copy of 128 rows, or, where the tile is half of that or less, in copies
// of 32 (rows behind the tile's last come along and are not looked at); others: four a copy (rows: a lane's).  The whole warp calls, one lane
// issues: a copy's operands have to be uniform, and where the compiler cannot see that they are it takes the lanes one by one (455 clocks a
// stage of two copies for 345).
struct RowMaps {
  CUtensorMap whole, part, row;        // boxes of 128, 32 and one row x 128 bytes
};
__device__ __forceinline__ uint32_t fetch_bytes(const LqAdTile& t) {
  return t.first < 0 ? (t.rows + 3) / 4 * 512 : 2 * t.rows > BM ? A_STAGE : (t.rows + 31) / 32 * 4096;
}
__device__ __forceinline__ void fetch_rows(uint32_t dst, const RowMaps& tm, int x, const LqAdTile& t, const int4& rows, uint32_t bar) {
  if (t.first < 0) {
    for (int i = 0; 4 * i < t.rows; ++i) {
      const int4 r = make_int4(__shfl_sync(0xffffffffu, rows.x, i), __shfl_sync(0xffffffffu, rows.y, i), __shfl_sync(0xffffffffu, rows.z, i),
                               __shfl_sync(0xffffffffu, rows.w, i));
      if (elect_one()) tma_gather4(dst + i * 512, &tm.row, x, r, bar);
    }
  } else if (2 * t.rows > BM) {
    if (elect_one()) tma_load_2d(dst, &tm.whole, x, t.first, bar);
  } else if (elect_one()) {
    for (int i = 0; 32 * i < t.rows; ++i) tma_load_2d(dst + i * 4096, &tm.part, x, t.first + 32 * i, bar);
  }
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm) {
  asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
}
__device__ __forceinline__ void prefetch_maps(const RowMaps& tm) {
  prefetch_map(&tm.whole); prefetch_map(&tm.part); prefetch_map(&tm.row);
}

// ---- down ----------------------------------------------------------------------------------------------------------
constexpr int DOWN_WARPS = 8;

struct DownParams {
  const LqAdTile* tiles;
  const int *ntiles, *perm;
  const LqAdMeta* meta;
  __half* T;
  float* rscale;
  int32_t* status;
  int* ready;
  int rp, k_stages, ring, tmem_cols, M;
};

// One tile of a cluster at a time, K / (64 SPLIT) stages a CTA.  Warp 0 fetches, warp 1 issues the MMAs into 128 x rp of tensor memory; then
// all warps bring the partial sums to shared memory and each CTA adds up 128 / SPLIT rows from all of the cluster, always in the same order.
// A short kernel is a chain of latencies: nothing waits for what it does not need (an empty slot's tile is formed like another and left
// unread), the loads of a row's sums are all in flight together.  (8192 x 1152, rank 32, us from the dependency's end: tile known 0.6, copies
// asked for 1.5, sums complete 6.4, in shared memory of all 7.5, T written 8.8.)
template <int SPLIT>
__global__ void __launch_bounds__(32 * DOWN_WARPS) lq_adapters_down_kernel(const __grid_constant__ RowMaps tmX, const __grid_constant__ CUtensorMap tmDown,
                                                                           const __grid_constant__ DownParams p) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * MAX_STAGES + 1];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int stage_bytes = A_STAGE + p.rp * 128;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int part = blockIdx.x % SPLIT, clusters = gridDim.x / SPLIT;
  auto full = [&](int s) { return smem_u32(&bars[s]); };
  auto empty = [&](int s) { return smem_u32(&bars[MAX_STAGES + s]); };
  const uint32_t done = smem_u32(&bars[2 * MAX_STAGES]);
  if (threadIdx.x == 0) {
    for (int s = 0; s < MAX_STAGES; ++s) { mbar_init(full(s), 1); mbar_init(empty(s), 1); }
    mbar_init(done, 1);
    abort_flag = 0;
    mbar_init_fence();
    prefetch_maps(tmX); prefetch_map(&tmDown);
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_slot), p.tmem_cols);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  grid_dependency_wait();
  // All that came before is complete: the up kernel may read it as soon as it starts.  (A word, and not the start alone, tells it so: where
  // another thread has put a kernel on the stream between the two, that one's start lets the up kernel start.)
  if (blockIdx.x == 0 && threadIdx.x == 96) st_release(p.ready, 1);
  grid_launch_dependents();

  // (a tile behind the last one holds anything: it is asked for together with their number, which saves a trip)
  LqAdTile tile = p.tiles[blockIdx.x / SPLIT];
  const int ntiles = lq_ad_tiles_of<false>(p.ntiles, p.M, p.status);
  const int k0 = part * p.k_stages / SPLIT, n = (part + 1) * p.k_stages / SPLIT - k0;
  bool ok = true;                                         // (a CTA that has given up still meets the others at their barriers)
  int used = 0;                                           // stages of the tiles before
#pragma unroll 1
  for (int ti = blockIdx.x / SPLIT, turn = 0; ti < ntiles; ti += clusters) {
    if (ti >= clusters) tile = p.tiles[ti];
    if (tile.adapter < 0) continue;                       // (the same for the whole cluster)
    const float scale = p.meta[tile.adapter].scale;
    if (warp == 0 && ok) {
      const uint32_t bytes = fetch_bytes(tile) + p.rp * 128;
      int4 rows = make_int4(0, 0, 0, 0);
      if (tile.first < 0) rows = tile_rows4(p.perm + tile.begin, tile.rows, lane);
      int it = used;
      for (; it < used + n; ++it) {
        const int s = it % p.ring;
        if (it >= p.ring && !(ok = mbar_wait_warp(empty(s), ((it / p.ring) & 1) ^ 1, &abort_flag, p.status, LQ_STAGE_PRODUCER))) break;
        const uint32_t a = base + s * stage_bytes;
        const int x = (k0 + it - used) * 128;             // bytes along K
        if (elect_one()) {
          mbar_expect_tx(full(s), bytes);
          tma_load_2d(a + A_STAGE, &tmDown, x, tile.adapter * p.rp, full(s));
        }
        __syncwarp();
        fetch_rows(a, tmX, x, tile, rows, full(s));
      }
      if (!ok)                                            // copies in flight land before the CTA goes
        for (int i = max(0, it - p.ring); i < it; ++i) mbar_settle(full(i % p.ring), (i / p.ring) & 1);
    } else if (warp == 1 && ok) {
      const uint32_t idesc = IDESC_F16 | idesc_shape(p.rp);
      for (int it = used; it < used + n; ++it) {
        const int s = it % p.ring;
        if (!(ok = mbar_wait_warp(full(s), (it / p.ring) & 1, &abort_flag, p.status, LQ_STAGE_MMA))) break;
        tc_fence_after();
        const uint64_t a = make_smem_desc(base + s * stage_bytes), b = make_smem_desc(base + s * stage_bytes + A_STAGE);
        if (elect_one()) {
#pragma unroll
          for (int k = 0; k < 4; ++k) tc_mma<TC_F16>(tmem, a + 2 * k, b + 2 * k, idesc, it > used || k != 0);
          tc_commit(empty(s));
          if (it + 1 == used + n) tc_commit(done);
        }
        __syncwarp();
      }
    }
    __syncwarp();
    if (ok) ok = mbar_wait(done, turn, &abort_flag, p.status, LQ_STAGE_DRAIN);
    ok = __syncthreads_and(ok && !abort_flag) != 0;
    used += n;
    turn ^= 1;
    // partial sums -> shared memory, rows 16 bytes longer than they are so that neighbouring rows lie in different banks; the ring is free:
    // the MMAs have read it
    const int pitch = p.rp + 4;
    if (ok) {
      tc_fence_after();
      const uint32_t row = base + (uint32_t)((warp & 3) * 32 + lane) * pitch * 4;
      for (int c = 16 * (warp >> 2); c < p.rp; c += 32) {
        uint32_t v[16];
        tmem_ld_32x16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + c, v);
        tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 4; ++j) sts_v4(row + (c + 4 * j) * 4, make_uint4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]));
      }
    }
    if constexpr (SPLIT > 1) cluster_sync();
    else __syncthreads();
    // eight threads to a row, a float4 in 32 columns each
    constexpr int ROWS = BM / SPLIT, AT_ONCE = 4 * DOWN_WARPS;
    const int j0 = threadIdx.x & 7;
#pragma unroll 1
    for (int r = threadIdx.x >> 3; ok && r < ROWS; r += AT_ONCE) {
      const int row = part * ROWS + r;
      float4 v[4];
      float top = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        v[q] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (4 * j0 + 32 * q < p.rp) {
          const uint32_t at = base + (uint32_t)(row * pitch + 4 * j0 + 32 * q) * 4;
          if constexpr (SPLIT == 1) {
            const uint4 u = lds_v4(at);
            v[q] = make_float4(__uint_as_float(u.x), __uint_as_float(u.y), __uint_as_float(u.z), __uint_as_float(u.w));
          } else {
            float4 u[SPLIT];
#pragma unroll
            for (int w = 0; w < SPLIT; ++w) u[w] = ld_peer_v4(peer_smem(at, w));
#pragma unroll
            for (int w = 0; w < SPLIT; ++w) { v[q].x += u[w].x; v[q].y += u[w].y; v[q].z += u[w].z; v[q].w += u[w].w; }
          }
        }
        top = fmaxf(fmaxf(top, fmaxf(fabsf(v[q].x), fabsf(v[q].y))), fmaxf(fabsf(v[q].z), fabsf(v[q].w)));
      }
#pragma unroll
      for (int d = 1; d < 8; d *= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
      if (row < tile.rows) {
        const int e = lq_ad_exponent(top);
        const float f = __int_as_float((127 + e) << 23);  // 2^e, |e| <= 100
        __half* to = p.T + (size_t)(tile.begin + row) * LQ_AD_TROW + 4 * j0;
        if (j0 == 0) p.rscale[tile.begin + row] = ldexpf(scale, -e);
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (4 * j0 + 32 * q < p.rp) {
            const float u[4] = {v[q].x * f, v[q].y * f, v[q].z * f, v[q].w * f};
            float lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) lo[i] = u[i] - __half2float(__float2half_rn(u[i]));
            *reinterpret_cast<uint2*>(to + 32 * q) = make_uint2(pack_halves(u[0], u[1]), pack_halves(u[2], u[3]));
            *reinterpret_cast<uint2*>(to + LQ_AD_TROW / 2 + 32 * q) = make_uint2(pack_halves(lo[0], lo[1]), pack_halves(lo[2], lo[3]));
          }
      }
    }
    // the others have read this CTA's sums; what follows may write over them, copies too
    if (ti + clusters < ntiles) {
      fence_proxy_async();
      tc_fence_before();
      if constexpr (SPLIT == 1) __syncthreads();
    }
    if constexpr (SPLIT > 1) cluster_sync();
    tc_fence_after();
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, p.tmem_cols);
  }
}

// ---- up ------------------------------------------------------------------------------------------------------------
constexpr int UP_DRAIN_WARPS = 16, UP_FIRST_DRAIN = 4, UP_THREADS = 32 * (UP_FIRST_DRAIN + UP_DRAIN_WARPS), UP_COLS = 128;
constexpr int PIECE = BM * 128, Y_SLOTS = 6;              // 128 rows x 128 bytes
__host__ __device__ constexpr int up_t_bufs(int na) { return na == 1 ? 2 : 1; }
__host__ __device__ constexpr int up_b_stages(int na) { return na == 1 ? 3 : 2; }
constexpr int up_smem(int na) { return 1024 + (2 * na * up_t_bufs(na) + na * up_b_stages(na) + Y_SLOTS) * PIECE; }

struct UpParams {
  const LqAdTile* tiles;
  const int *ntiles, *perm;
  const LqAdMeta* meta;
  const float* rscale;
  void* Y;
  int32_t* status;
  int* ready;
  int N, Npad, chunks, in_place, M;
};

// Persistent, one CTA an SM: the steps (tile, 128 columns) of all tiles are cut into runs of like length.  Warp 0 fetches a tile's T (both
// halves) and each step's slab of B, warp 1 issues hi B + lo B into one of two accumulators, warp 2 fetches Y0 into a ring of 96 KB, pieces
// of 128 rows x 128 bytes; the drain warps hold 32 rows x 32 columns each: they add, round and store.  B's rows lie in the order that gives a
// lane eight neighbouring columns.
// 8192 x 3456, rank 32: 20 us from the down kernel's end on, 17.3 at the measured copy rate (Y0 straight into registers a step ahead, 32 KB in
// flight: 30.7).  Both kernels and the map, us in a graph of ten passes: 8192 rows 1152 x 3456, rank 32 37; 32768 rows 5600 x 2240, rank 128 140 to 142
// (103 at the copy rate), in long runs 155 to 168.
template <bool F32, int NA>      // NA: 64-wide pieces of the rank
__global__ void __launch_bounds__(UP_THREADS, 1) lq_adapters_up_kernel(const __grid_constant__ CUtensorMap tmT, const __grid_constant__ CUtensorMap tmUp,
                                                                       const __grid_constant__ RowMaps tmY,
                                                                       const __grid_constant__ UpParams p) {
  constexpr int NT = up_t_bufs(NA), NB = up_b_stages(NA), T_BUF = 2 * NA * PIECE, B_STAGE = NA * PIECE, B_AT = NT * T_BUF, Y_AT = B_AT + NB * B_STAGE;
  // Pieces of a step, and warps that wait for one and give it back.  A wait tells a phase from the next one, not from the one after that, so
  // who waits on a place of the ring has to wait for each of its turns.  With two pieces a step the six places are always read by the same
  // warps.  With four a place's turns would alternate between two groups of them: every warp waits for all pieces and gives all back.
  constexpr int YP = F32 ? 4 : 2, Y_READERS = F32 ? UP_DRAIN_WARPS : UP_DRAIN_WARPS / YP;
  static_assert(F32 || Y_SLOTS % YP == 0, "");
  extern __shared__ unsigned char smem_raw[];
  enum { TFULL = 0, TFREE = NT, BFULL = 2 * NT, BFREE = BFULL + NB, AFULL = BFREE + NB, YFULL = AFULL + 2, AFREE = YFULL + Y_SLOTS };
  enum { YFREE = AFREE + 2, NBAR = YFREE + Y_SLOTS };
  __shared__ __align__(8) uint64_t bars[NBAR];
  __shared__ uint32_t tmem_slot;
  __shared__ volatile int abort_flag;
  __shared__ int early;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  auto bar = [&](int i) { return smem_u32(&bars[i]); };
  if (threadIdx.x == 0) {
    for (int i = 0; i < NBAR; ++i) mbar_init(bar(i), i >= YFREE ? Y_READERS : i >= AFREE ? UP_DRAIN_WARPS : 1);
    abort_flag = 0;
    mbar_init_fence();
    prefetch_map(&tmT); prefetch_map(&tmUp); prefetch_maps(tmY);
  }
  if (warp == 1) tmem_alloc(smem_u32(&tmem_slot), 2 * UP_COLS);
  if (threadIdx.x == 96) early = ld_acquire(p.ready);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  grid_launch_dependents();
  // Where the down kernel has said that all that came before it has completed, the map, the factors and Y0 are there, and only T and its
  // rows' scales are waited for (and every CTA waits, so that who waits for this kernel has waited for that one).  Else everything is.
  if (warp == 3 || !early) grid_dependency_wait();

  const int ntiles = lq_ad_tiles_of<false>(p.ntiles, p.M, p.status);
  const long long total = (long long)ntiles * p.chunks;
  const long long lo = total * blockIdx.x / gridDim.x, hi = total * (blockIdx.x + 1) / gridDim.x;
  const int n = (int)(hi - lo), ti0 = (int)(lo / p.chunks), ch0 = (int)(lo - (long long)ti0 * p.chunks);
  // a tile and the rank of its adapter; every role reads those of the next tile while it is busy with one
  struct Info {
    LqAdTile tile;
    int rank;
  };
  const auto info = [&](int ti) {
    Info f = {{-1, 0, 0, -1}, 0};
    if (ti < ntiles) {
      f.tile = p.tiles[ti];
      if (f.tile.adapter >= 0) f.rank = p.meta[f.tile.adapter].rank;
    }
    return f;
  };
  bool ok = true;

  if (warp == 0) {
    if (n > 0) {
      int t_uses = 0, b_uses = 0;
      Info f = info(ti0), next = info(ti0 + 1);
      bool enter = true;
      for (int i = 0, ti = ti0, ch = ch0; i < n && ok; ++i) {
        const int pieces = (f.rank + 63) / 64;
        if (f.rank > 0) {
          const int s = b_uses % NB;
          if (b_uses >= NB && !(ok = mbar_wait_warp(bar(BFREE + s), ((b_uses / NB) & 1) ^ 1, &abort_flag, p.status, LQ_STAGE_PRODUCER))) break;
          if (elect_one()) {
            mbar_expect_tx(bar(BFULL + s), pieces * PIECE);
            for (int a = 0; a < pieces; ++a)
              tma_load_2d(base + B_AT + s * B_STAGE + a * PIECE, &tmUp, 128 * a, f.tile.adapter * p.Npad + UP_COLS * ch, bar(BFULL + s));
          }
          __syncwarp();
          ++b_uses;
        }
        if (enter && f.rank > 0) {
          const int buf = t_uses % NT;
          if (t_uses == 0) grid_dependency_wait();
          if (t_uses >= NT && !(ok = mbar_wait_warp(bar(TFREE + buf), ((t_uses / NT) & 1) ^ 1, &abort_flag, p.status, LQ_STAGE_PRODUCER))) break;
          if (elect_one()) {
            mbar_expect_tx(bar(TFULL + buf), 2 * pieces * PIECE);
            for (int a = 0; a < pieces; ++a) {
              tma_load_2d(base + buf * T_BUF + a * PIECE, &tmT, 128 * a, f.tile.begin, bar(TFULL + buf));
              tma_load_2d(base + buf * T_BUF + (NA + a) * PIECE, &tmT, LQ_AD_TROW + 128 * a, f.tile.begin, bar(TFULL + buf));
            }
          }
          __syncwarp();
          ++t_uses;
        }
        enter = ++ch == p.chunks;
        if (enter) {
          ch = 0;
          f = next;
          next = info(++ti + 1);
        }
      }
      if (!ok && lane == 0) {                             // copies in flight land before the CTA goes
        for (int u = max(0, t_uses - NT); u < t_uses; ++u) mbar_settle(bar(TFULL + u % NT), (u / NT) & 1);
        for (int u = max(0, b_uses - NB); u < b_uses; ++u) mbar_settle(bar(BFULL + u % NB), (u / NB) & 1);
      }
    }
  } else if (warp == 1) {
    if (n > 0) {
      int t_uses = 0, b_uses = 0;
      Info f = info(ti0), next = info(ti0 + 1);
      bool enter = true;
      constexpr uint32_t idesc = IDESC_F16 | idesc_shape(UP_COLS);
      for (int i = 0, ti = ti0, ch = ch0; i < n && ok; ++i) {
        if (enter && f.rank > 0) {
          ok = mbar_wait_warp(bar(TFULL + t_uses % NT), (t_uses / NT) & 1, &abort_flag, p.status, LQ_STAGE_MMA);
          ++t_uses;
        }
        if (f.rank > 0 && ok) {
          const int s = b_uses % NB, acc = b_uses & 1, buf = (t_uses - 1) % NT;
          if (b_uses >= 2) ok = mbar_wait_warp(bar(AFREE + acc), ((b_uses >> 1) & 1) ^ 1, &abort_flag, p.status, LQ_STAGE_MMA);
          ok = ok && mbar_wait_warp(bar(BFULL + s), (b_uses / NB) & 1, &abort_flag, p.status, LQ_STAGE_MMA);
          if (!ok) break;
          tc_fence_after();
          const int steps = (f.rank + 15) / 16;
          const uint64_t hi = make_smem_desc(base + buf * T_BUF), lo = make_smem_desc(base + buf * T_BUF + NA * PIECE);
          const uint64_t slab = make_smem_desc(base + B_AT + s * B_STAGE);
          if (elect_one()) {
            for (int k = 0; k < steps; ++k) {             // (64 of the rank are a piece)
              const uint32_t at = (uint32_t)((k >> 2) * (PIECE >> 4) + 2 * (k & 3));
              tc_mma<TC_F16>(tmem + acc * UP_COLS, hi + at, slab + at, idesc, k != 0);
              tc_mma<TC_F16>(tmem + acc * UP_COLS, lo + at, slab + at, idesc, 1);
            }
            tc_commit(bar(BFREE + s));
            tc_commit(bar(AFULL + acc));
            if (i + 1 == n || ch + 1 == p.chunks) tc_commit(bar(TFREE + buf));
          }
          __syncwarp();
          ++b_uses;
        }
        enter = ++ch == p.chunks;
        if (enter) {
          ch = 0;
          f = next;
          next = info(++ti + 1);
        }
      }
    }
  } else if (warp == 2) {
    if (n > 0) {
      int uses = 0;
      Info f = info(ti0), next = info(ti0 + 1);
      int4 rows = make_int4(0, 0, 0, 0);
      bool enter = true;
      for (int i = 0, ti = ti0, ch = ch0; i < n && ok; ++i) {
        if (f.rank > 0 || !p.in_place) {                  // (rows without an adapter are copied, or left alone)
          if (enter && f.tile.first < 0) rows = tile_rows4(p.perm + f.tile.begin, f.tile.rows, lane);
          for (int u = 0; u < YP && ok; ++u, ++uses) {
            const int s = uses % Y_SLOTS, x = (ch * YP + u) * 128;
            if (uses >= Y_SLOTS && !(ok = mbar_wait_warp(bar(YFREE + s), ((uses / Y_SLOTS) & 1) ^ 1, &abort_flag, p.status, LQ_STAGE_PRODUCER))) break;
            if (elect_one()) mbar_expect_tx(bar(YFULL + s), fetch_bytes(f.tile));
            __syncwarp();
            fetch_rows(base + Y_AT + s * PIECE, tmY, x, f.tile, rows, bar(YFULL + s));
          }
        }
        enter = ++ch == p.chunks;
        if (enter) {
          ch = 0;
          f = next;
          next = info(++ti + 1);
        }
      }
      if (!ok && lane == 0)
        for (int u = max(0, uses - Y_SLOTS); u < uses; ++u) mbar_settle(bar(YFULL + u % Y_SLOTS), (u / Y_SLOTS) & 1);
    }
  } else if (warp >= UP_FIRST_DRAIN && n > 0) {
    // ---------------------------------------------------------------------- drain
    const int quad = warp & 3, cq = (warp - UP_FIRST_DRAIN) >> 2, g = lane >> 2, t = lane & 3;
    const uint32_t tlane = tmem + ((uint32_t)(quad * 32) << 16) + 32 * cq;
    constexpr int YW = F32 ? 2 : 1;                       // 16-byte words of a lane's eight columns
    // place of the lane's word w of row g + 8 q in a piece: its 128-byte rows are swizzled by 16 bytes
    const int unit = F32 ? cq : cq >> 1, word = F32 ? 2 * t : 4 * (cq & 1) + t;
    const uint32_t y_row = base + Y_AT + (uint32_t)(quad * 32 + g) * 128;
    struct Rows {
      int row[4];                                         // -1: none
      float scale[4];
      int rank, rows;
    };
    bool waited = false;
    const auto rows_of = [&](int ti) {
      const Info f = info(ti);
      if (!waited) grid_dependency_wait();
      waited = true;
      Rows r;
      r.rank = f.rank;
      r.rows = f.tile.rows;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = quad * 32 + g + 8 * i;
        const bool in = at < f.tile.rows;
        r.row[i] = in ? p.perm[f.tile.begin + at] : -1;
        r.scale[i] = in && f.tile.adapter >= 0 ? p.rscale[f.tile.begin + at] : 0.f;
      }
      return r;
    };
    int uses = 0, y_uses = 0;
    Rows r = rows_of(ti0), r_next = {};
    for (int i = 0, ti = ti0, ch = ch0; i < n; ++i) {
      const bool last = ch + 1 == p.chunks;
      if (last && i + 1 < n) r_next = rows_of(ti + 1);
      if (r.rank > 0 || !p.in_place) {
        const int s = (y_uses + unit) % Y_SLOTS;
        bool landed = true;
        for (int u = F32 ? 0 : unit; landed && u < (F32 ? YP : unit + 1); ++u) {
          const int use = y_uses + u;
          landed = mbar_wait_warp(bar(YFULL + use % Y_SLOTS), (use / Y_SLOTS) & 1, &abort_flag, p.status, LQ_STAGE_DRAIN);
        }
        if (!landed) break;
        const int acc = uses & 1;
        if (r.rank > 0) {
          if (!mbar_wait_warp(bar(AFULL + acc), (uses >> 1) & 1, &abort_flag, p.status, LQ_STAGE_DRAIN)) break;
          ++uses;
          tc_fence_after();
        }
        const int c = ch * UP_COLS + 32 * cq + 8 * t;
        // rows g, g + 8, then rows g + 16, g + 24 of the quarter, where the tile has some: fragment registers 4 j .. 4 j + 3 hold row g,
        // columns 2 j, 2 j + 1 of this lane's eight, then row g + 8 the same columns
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const bool any = 32 * quad + 16 * h < r.rows;
          uint32_t v[16];
          uint4 y[2][YW];
          if (any) {
            if (r.rank > 0) tmem_ld_16x256b_x4(tlane + ((uint32_t)(16 * h) << 16) + acc * UP_COLS, v);
#pragma unroll
            for (int q = 0; q < 2; ++q)
#pragma unroll
              for (int w = 0; w < YW; ++w) y[q][w] = lds_v4(y_row + s * PIECE + (2 * h + q) * 1024 + (((word + w) ^ g) << 4));
            if (r.rank > 0) tmem_ld_wait();
          }
          if (h == 1 && r.rank > 0) {                     // the accumulator is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(AFREE + acc));
          }
          if (any)
#pragma unroll
            for (int q = 0; q < 2; ++q)
              if (r.row[2 * h + q] >= 0 && c < p.N) {
                const float2 by = make_float2(r.scale[2 * h + q], r.scale[2 * h + q]);
                const size_t to = (size_t)(unsigned)r.row[2 * h + q] * (unsigned)p.N + c;
                const auto d = [&](int j) {               // columns 2 j, 2 j + 1
                  return make_float2(__uint_as_float(v[4 * j + 2 * q]), __uint_as_float(v[4 * j + 2 * q + 1]));
                };
                if constexpr (F32) {
                  float2* f = reinterpret_cast<float2*>(&y[q][0]);
                  if (r.rank > 0)                         // (a row without an adapter keeps its bits)
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = __ffma2_rn(by, d(j), f[j]);
                  uint4* at = reinterpret_cast<uint4*>(reinterpret_cast<float*>(p.Y) + to);
                  at[0] = y[q][0]; at[YW - 1] = y[q][YW - 1];
                } else {
                  __half2* f = reinterpret_cast<__half2*>(&y[q][0]);
                  if (r.rank > 0)
#pragma unroll
                    for (int j = 0; j < 4; ++j) f[j] = __float22half2_rn(__ffma2_rn(by, d(j), __half22float2(f[j])));
                  *reinterpret_cast<uint4*>(reinterpret_cast<__half*>(p.Y) + to) = y[q][0];
                }
              }
        }
        // (behind the stores, which have to wait for the words that they store: right behind its loads the arrival, and the next copy with
        // it, can overtake them)
        __syncwarp();
        if (lane < (F32 ? YP : 1)) mbar_arrive(bar(YFREE + (F32 ? (y_uses + lane) % Y_SLOTS : s)));
        y_uses += YP;
      }
      if (last) { r = r_next; ch = 0; ++ti; }
      else ++ch;
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem, 2 * UP_COLS);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.ready = 0;  // (a CTA that starts later than this waits, for nothing any more)
}

constexpr int DOWN_SMEM = 110 * 1024;                     // two CTAs an SM

template <int SPLIT>
cudaError_t launch_down(const lq_adapters* S, const lq_rowmap* R, const RowMaps& tmX, DownParams& d, cudaStream_t st) {
  const int stage = A_STAGE + S->rp * 128, most = (d.k_stages + SPLIT - 1) / SPLIT;
  d.ring = std::min(std::min(MAX_STAGES, most), (DOWN_SMEM - 1024) / stage);
  while (d.tmem_cols < S->rp) d.tmem_cols *= 2;
  const int smem = 1024 + std::max(d.ring * stage, BM * (S->rp + 4) * 4);
  // no more clusters than are resident: with many slots most tiles that there might be are not there (8192 x 1152 x 3456, rank 32, 1023 slots
  // of which eight are used, us with the map: 61.1 by a cluster for each, 40.4 so)
  const int tiles = std::min(lq_ad_tiles(R->M, R->slots, BM), std::max(1, 2 * R->sms / SPLIT));
  return lq_launch_cluster(lq_adapters_down_kernel<SPLIT>, tiles * SPLIT, 32 * DOWN_WARPS, SPLIT, smem, st, tmX, S->tmDown, d);
}

template <bool F32, int NA>
cudaError_t launch_up(const lq_adapters* S, const lq_rowmap* R, const RowMaps& tmY, const UpParams& p, cudaStream_t st) {
  const long long steps = (long long)lq_ad_tiles(R->M, R->slots, BM) * p.chunks;
  return lq_launch(lq_adapters_up_kernel<F32, NA>, (int)std::min<long long>(steps, R->sms), UP_THREADS, up_smem(NA), st, R->tmT, S->tmUp, tmY, p);
}

}  // namespace

lq_status lq_adapters_tiles_prepare() {
  const auto room = [](auto* kernel, int bytes) {
    return lq_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) == cudaSuccess;
  };
  return room(lq_adapters_down_kernel<1>, DOWN_SMEM) && room(lq_adapters_down_kernel<2>, DOWN_SMEM) &&
                 room(lq_adapters_down_kernel<4>, DOWN_SMEM) && room(lq_adapters_down_kernel<8>, DOWN_SMEM) &&
                 room(lq_adapters_up_kernel<false, 1>, up_smem(1)) && room(lq_adapters_up_kernel<true, 1>, up_smem(1)) &&
                 room(lq_adapters_up_kernel<false, 2>, up_smem(2)) && room(lq_adapters_up_kernel<true, 2>, up_smem(2))
             ? LQ_OK
             : LQ_ERR_CUDA;
}

lq_status lq_adapters_forward_tiles(const lq_adapters* S, const lq_rowmap* R, const void* X, const void* Y0, void* Y, lq_out_dtype dt, cudaStream_t st) {
  RowMaps tmX, tmY;
  const auto rows_of = [R](RowMaps* tm, const void* base, uint64_t bytes) {
    lq_status s;
    if ((s = lq_make_tmap_bytes(&tm->whole, const_cast<void*>(base), (uint64_t)R->M, bytes, BM)) != LQ_OK) return s;
    if ((s = lq_make_tmap_bytes(&tm->part, const_cast<void*>(base), (uint64_t)R->M, bytes, 32)) != LQ_OK) return s;
    return lq_make_tmap_bytes(&tm->row, const_cast<void*>(base), (uint64_t)R->M, bytes, 1);
  };
  lq_status s;
  if ((s = rows_of(&tmX, X, (uint64_t)S->K * 2)) != LQ_OK || (s = rows_of(&tmY, Y0, (uint64_t)S->N * (dt == LQ_OUT_F32 ? 4 : 2))) != LQ_OK) return s;
  int32_t* status = lq_device_status_ptr(S->device);
  if (!status) return LQ_ERR_CUDA;
  DownParams d = {R->d_tiles, R->d_ntiles, R->d_perm, S->d_meta, R->d_T, R->d_rscale, status, R->d_ntiles + 3, S->rp, lq_ceil_div(S->K, 64), 1, 32, R->M};
  // K is shared by as many CTAs as fill the SMs twice over, each with at least two stages (us with the map by 1, 2, 4 and 8 of them, 5600 x
  // 2240, rank 128: 4096 rows 60.2, 44.6, 38.9, 38.0; 8192 rows 70.0, 57.4, 53.9, 63.2; 16384 rows 88.4, 82.8, 91.6, 132; 32768 rows 142,
  // 150, 203, 289)
  const int tiles = lq_ceil_div(R->M, BM);
  int split = 1;
  while (split < 8 && tiles * 2 * split <= 2 * R->sms && d.k_stages >= 4 * split) split *= 2;
  cudaError_t e = split == 1   ? launch_down<1>(S, R, tmX, d, st)
                  : split == 2 ? launch_down<2>(S, R, tmX, d, st)
                  : split == 4 ? launch_down<4>(S, R, tmX, d, st)
                               : launch_down<8>(S, R, tmX, d, st);
  if (lq_note_cuda(e) != cudaSuccess) return LQ_ERR_CUDA;
  const UpParams u = {R->d_tiles, R->d_ntiles, R->d_perm, S->d_meta, R->d_rscale, Y, status, R->d_ntiles + 3,
                      S->N, S->Npad, lq_ceil_div(S->N, UP_COLS), Y0 == Y, R->M};
  if (dt == LQ_OUT_F32) e = S->rp <= 64 ? launch_up<true, 1>(S, R, tmY, u, st) : launch_up<true, 2>(S, R, tmY, u, st);
  else e = S->rp <= 64 ? launch_up<false, 1>(S, R, tmY, u, st) : launch_up<false, 2>(S, R, tmY, u, st);
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
