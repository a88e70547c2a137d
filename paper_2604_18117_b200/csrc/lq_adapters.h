// Low-rank adapters: the handles and what the two forms of the forward share (lq_adapters.cu, lq_adapters_tile.cu).
#pragma once

#include <cuda_fp16.h>

#include "lq_internal.h"

// A map's rows are cut into tiles of rows of one adapter: 16 rows for the form that serves few rows, 128 for the one that serves many.
constexpr int LQ_AD_SMALL_M = 256, LQ_AD_SMALL_TILE = 16, LQ_AD_TILE = 128;
constexpr int LQ_AD_TROW = 256;        // halves of a row of the intermediate: 128 hi, 128 lo

struct LqAdTile {
  int adapter, begin, rows, first;     // adapter -1: none; rows are perm[begin] .. perm[begin + rows - 1]; first: perm[begin] where the
                                       // rows are neighbours, else -1
};
struct LqAdMeta {
  int rank;                            // 0: empty slot
  float scale;
};

struct lq_adapters {
  int K, N, Npad, max_rank, rp, slots, device;  // rp: ranks are stored in rows of so many (16, or a multiple of 32); Npad: N rounded up to 32
  __half* d_down;                      // [slots][rp][K]     column j of A as a row
  __half* d_up;                        // [slots][Npad][rp]  column n of B as row lq_col32_slot(n)
  LqAdMeta* d_meta;                    // [slots]
  CUtensorMap tmDown, tmUp;            // boxes of [rp] and [128] rows x 128 bytes, 128-byte swizzle
};
struct lq_rowmap {
  int M_max, slots, device, M, tile_rows, tiles_max, sms;
  int* d_ntiles;
  LqAdTile* d_tiles;                   // [tiles_max]
  int* d_perm;                         // [M_max]
  __half* d_T;                         // [M_max + 128][LQ_AD_TROW], in the order of perm (only with M_max > LQ_AD_SMALL_M)
  float* d_rscale;                     // [M_max + 128] what a row of T times B is multiplied with
  CUtensorMap tmT;
};

// most tiles that M rows can make
static inline int lq_ad_tiles(const lq_rowmap* R) { return R->M < lq_ceil_div(R->M, R->tile_rows) + R->slots ? R->M : lq_ceil_div(R->M, R->tile_rows) + R->slots; }

lq_status lq_adapters_forward_tiles(const lq_adapters* S, const lq_rowmap* R, const void* X, const void* Y0, void* Y, lq_out_dtype dt, cudaStream_t st);
lq_status lq_adapters_tiles_prepare();   // once for each device that a map is made on, with that device current

#ifdef __CUDACC__
// The power of two that brings a row's largest magnitude to [2^14, 2^15): no half overflows, and hi + lo keep 22 bits of it.
__device__ __forceinline__ int lq_ad_exponent(float top) {
  int e = 0;
  if (top > 0.f && top < INFINITY) frexpf(top, &e);
  return max(-100, min(100, 15 - e));
}
#endif
