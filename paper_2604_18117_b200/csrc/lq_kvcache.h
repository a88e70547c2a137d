// The cache of keys and values: its handle, how it lies in memory, and how a step's sequences are found in it (lq_kvcache.cu, lq_attn.cu,
// lq_attn_tile.cu).
#pragma once

#include <cuda_fp16.h>

#include "lq_heads_places.h"
#include "lq_internal.h"
#include "lq_kv_rows.h"

// A record holds 32 tokens of one head: 32 bytes that begin with the exponents of keys and values, the keys, the values.  Codes are kept as
// bytes u = c + 128, in the order in which a warp of the attention kernels reads them as operands of m16n8k16 products, 16 bytes a lane
// (c8 = lane / 4, t = lane % 4) for every 16 entries of the head:
//   keys    word i = 2 s + h: token lq_kv_token(c8, i), bytes: entries 4 t .. 4 t + 3 of the 16 (column c8 of the products' tile i)
//   values  word 2 s + i: entry 2 c8 + i of the 16, bytes: tokens 16 s + 4 t .. 4 t + 3
// so that every load is one of 16 bytes a lane, neighbours across lanes, no byte has to change lanes, and stores of opened codes to swizzled
// rows of 128 bytes meet in no bank.  Records follow each other by layer, page, block of the page and head.
constexpr int LQ_KV_HEAD = 32, LQ_KV_E_MIN = -20, LQ_KV_E_MAX = 9;
static inline __host__ __device__ int lq_kv_side_bytes(int Dp) { return LQ_KV_BLOCK * Dp; }
static inline __host__ __device__ int lq_kv_record_bytes(int Dp) { return LQ_KV_HEAD + 2 * lq_kv_side_bytes(Dp); }
static inline __host__ __device__ int lq_kv_token(int c8, int i) { return 16 * (i >> 1) + 4 * (c8 >> 1) + 2 * (c8 & 1) + (i & 1); }

// heads are stored padded to the next of these
constexpr int LQ_KV_DIMS[] = {64, 80, 96, 112, 128, 192, 256};
static inline int lq_kv_padded(int D) {
  for (int d : LQ_KV_DIMS)
    if (D <= d) return d;
  return 0;
}

constexpr int LQ_ATTN_ROWS = 16;         // rows (new tokens x query heads of a group) of a tile of the form for few rows
struct lq_kvcache {
  int layers, pages, page_tokens, heads, D, Dp, device, sms;
  uint8_t* d_records;
  // workspace of the attention: for each block of its grid two partial results of a tile of rows, and a count of those that have arrived
  float* d_part;                         // [2 * sms][LQ_ATTN_ROWS][Dp + 4]: maximum, sum, -, -, sums
  int* d_count;                          // [sms]
  float* d_tile_part;                    // the same for tiles of 256 rows (Dp <= 128)
  int4* d_tile_meta;
};

// A step's sequences, as kernels take them
struct LqBatch {
  const int32_t *row_start, *length, *pages;
  int sequences, rows, each;             // each: rows of every sequence where row_start is NULL
  int page_stride, page_count, page_blocks, heads;
  long long record;                      // bytes
  uint64_t by_page_blocks;               // 2^37 / page_blocks, rounded up: quotients of what is below 2^26 (page_blocks <= 2^11)
};

// checks a caller's batch against a cache; LQ_OK fills *out
lq_status lq_take_batch(const lq_kvcache* C, int32_t layer, const lq_kvbatch* b, LqBatch* out);
// whether an output lies on a batch's arrays, which blocks of a launch still read while others write theirs: lengths, pages, and
// `entries` entries of one more (which may be NULL)
LqPlaces lq_batch_meets(const LqBatch& b, const int32_t* more, int entries, const LqRuns& out);
static inline uint8_t* lq_kv_layer(const lq_kvcache* C, int layer) {
  return C->d_records + (size_t)layer * C->pages * (C->page_tokens / LQ_KV_BLOCK) * C->heads * lq_kv_record_bytes(C->Dp);
}
lq_status lq_attn_prepare(const lq_kvcache* C);        // once for each cache, with its device current
lq_status lq_attn_tile_prepare(const lq_kvcache* C);

#ifdef __CUDACC__
// Rows of a sequence and its tokens.  What the arrays hold is the caller's: rows are kept within the call's, so that nothing outside its
// tensors is touched.
struct LqSeq {
  int row, n, len;                       // first row, rows, tokens with them
};
__device__ __forceinline__ LqSeq lq_seq(const LqBatch& b, int s) {
  LqSeq q;
  if (b.row_start) {
    const LqRowRange r = lq_kv_rows(b.row_start[s], b.row_start[s + 1], b.rows);
    q.row = r.row;
    q.n = r.n;
  } else {
    q.row = s * b.each;
    q.n = b.each;
  }
  q.len = b.length[s];
  return q;
}
// Whether a sequence's length fits its row of pages.  A kernel that meets another says so in the status word and leaves the sequence out.
__device__ __forceinline__ bool lq_seq_fits(const LqBatch& b, const LqSeq& q) {
  return q.len >= 0 && ((long long)q.len + LQ_KV_BLOCK - 1) / LQ_KV_BLOCK <= (long long)b.page_stride * b.page_blocks;
}
__device__ __forceinline__ void lq_kv_refuse(int32_t* status) {
  if (atomicCAS(status, 0, (int)LQ_ERR_INVALID_ARG) == 0) status[1] = LQ_STAGE_NONE;
}
__device__ __forceinline__ int lq_kv_slot(const LqBatch& b, int block) { return (int)(((uint64_t)(uint32_t)block * b.by_page_blocks) >> 37); }
// index of a block's first record (of head 0), or -1: the page is none of the cache's
__device__ __forceinline__ long long lq_kv_at(const LqBatch& b, int block, int slot, int page) {
  if (page < 0 || page >= b.page_count) return -1;
  return ((long long)page * b.page_blocks + (block - slot * b.page_blocks)) * b.heads;
}
__device__ __forceinline__ long long lq_kv_at(const LqBatch& b, int s, int block) {
  const int slot = lq_kv_slot(b, block);
  return lq_kv_at(b, block, slot, b.pages[(long long)s * b.page_stride + slot]);
}
// Two codes of a word (SEL: 0x4140 the lower two, 0x4342 the upper two, 0x4240 and 0x4341 every second one) as halves, each times 2^(e - 4): a byte u under the upper byte `high` of a
// half is (1024 + u) 2^(e - 4), and what `less` takes off leaves u - 128 = c of that, all of it exact for e in [-20, 9].
__device__ __forceinline__ uint32_t lq_kv_high(int e) { return 0x01010101u * (uint32_t)(0x64 + 4 * (e - 4)); }
__device__ __forceinline__ __half2 lq_kv_less(uint32_t high) {          // 1152 2^(e - 4) = 1024 2^(e - 4) + 128 2^(e - 4)
  const uint32_t h = ((high & 0xFF) << 8) | 0x80;
  const uint32_t w = h | (h << 16);
  return *reinterpret_cast<const __half2*>(&w);
}
template <uint32_t SEL>
__device__ __forceinline__ uint32_t lq_kv_open(uint32_t word, uint32_t high, __half2 less) {
  const uint32_t w = __byte_perm(word, high, SEL);
  const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&w), less);
  return *reinterpret_cast<const uint32_t*>(&v);
}
#endif
