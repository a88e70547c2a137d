// Low-rank adapters: the handles and what the two forms of the forward share (lq_adapters.cu, lq_adapters_tile.cu).
#pragma once

#include <cuda_fp16.h>

#include "lq_internal.h"

// Two forms of the forward: one of clusters on tiles of 16 rows of one adapter, for few rows of narrow factors, and one on tiles of 128 rows.
// us with the map, K x N and rank, small / large form.  Six requests of neighbouring rows: 1152 x 3456, 32: 600 rows 14.1 / 15.5, 1400 rows
// 18.2 / 17.7, 2048 rows 19.0 / 19.6; 512 x 8192, 64: 90 rows 14.3 / 15.2, 250 rows 20.7 / 15.9.  Rows in any order, which the large form
// fetches four at a time: 1160 x 2312, 24, 1365 rows 16.8 / 23.9 (fp32 21.2 / 31.9); so such rows take a step up at the cut, which goes by their
// number alone (1536 and 1537 rows 17.6 and 24.6, fp32 22.0 and 33.0; neighbours 16.9 and 17.8, 21.3 and 21.5).  Rows with an adapter each:
// 512 x 8192, 64: 64 rows 27.8 / 34.8.  Ranks above 64 (the small form is not built for them): 5600 x 2240, 128: one row 23.9 / 17.2, 12 rows
// 26.8 / 22.3; 512 x 8192, 128: one row 20.0 / 12.7; 1152 x 1152, 96: one row 12.4 / 13.2, the one where the small form was ahead.
constexpr int LQ_AD_SMALL_TILE = 16, LQ_AD_TILE = 128;
constexpr int LQ_AD_SMALL_M = 1536, LQ_AD_SMALL_M_64 = 128;      // most rows of the small form, for stored ranks up to 32, 64
static inline bool lq_ad_small_form(int M, int rp) { return rp <= 32 ? M <= LQ_AD_SMALL_M : rp <= 64 && M <= LQ_AD_SMALL_M_64; }
constexpr int LQ_AD_ANY_M = 16;        // maps of so few rows do not look for neighbours: at most four copies bring a tile's rows
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
  int M_max, slots, device, M, sms;
  int* d_ntiles;                       // [4]: tiles of 128 rows, of 16, rows that were sorted, 1 from a down kernel's wait to its up kernel's end
  LqAdTile *d_tiles, *d_small;         // (tiles of 16 rows only up to LQ_AD_SMALL_M rows)
  int* d_perm;                         // [M_max]
  __half* d_T;                         // [M_max + 128][LQ_AD_TROW], in the order of perm
  float* d_rscale;                     // [M_max + 128] what a row of T times B is multiplied with
  CUtensorMap tmT;
};

// most tiles that M rows can make
static inline int lq_ad_tiles(int M, int slots, int rows) { return M < lq_ceil_div(M, rows) + slots ? M : lq_ceil_div(M, rows) + slots; }

lq_status lq_adapters_forward_tiles(const lq_adapters* S, const lq_rowmap* R, const void* X, const void* Y0, void* Y, lq_out_dtype dt, cudaStream_t st);
lq_status lq_adapters_tiles_prepare();   // once for each device that a map is made on, with that device current

#ifdef __CUDACC__
// The tiles (of 128 rows, or of 16) of a forward of M rows.  None where the map holds other rows by now, so that no row behind the forward's
// is touched: a graph that sorts was replayed between, or was captured and not yet replayed.  A forward that finds that says so in the status
// word.
template <bool SMALL>
__device__ __forceinline__ int lq_ad_tiles_of(const int* d_ntiles, int M, int32_t* status) {
  const int4 n = *reinterpret_cast<const int4*>(d_ntiles);
  if (n.z == M) return SMALL ? n.y : n.x;
  if (blockIdx.x == 0 && threadIdx.x == 0 && atomicCAS(status, 0, (int)LQ_ERR_INVALID_ARG) == 0) status[1] = LQ_STAGE_NONE;
  return 0;
}

// The power of two that brings a row's largest magnitude to [2^14, 2^15): no half overflows, and hi + lo keep 22 bits of it.
__device__ __forceinline__ int lq_ad_exponent(float top) {
  int e = 0;
  if (top > 0.f && top < INFINITY) frexpf(top, &e);
  return max(-100, min(100, 15 - e));
}
#endif
