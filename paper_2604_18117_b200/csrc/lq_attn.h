// Attention over the cache: what its two forms share (lq_attn.cu, lq_attn_tile.cu).
#pragma once

#include "lq_kvcache.h"

struct LqAttnParams {
  LqBatch b;
  const uint8_t* records;
  const __half* q;
  __half* out;
  long long q_row, q_head, out_row, out_head;
  int D, group;                          // query heads of a head of keys and values
  int causal, window, sinks;
  float scale;                           // of the products of queries and stored keys, times log2 e
  float* part;
  int* count;
  int few, many;                         // sequences whose rows * group are in [few, many) are this launch's
  int whole, splits;                     // form for many rows: tiles with a thread block each; blocks that share out the tokens of each of the others
  float* tile_part;                      // [sms][Dp + 2][256]: what each of them leaves: sums by entry, maxima, sums of weights
  int4* tile_meta;                       // [sms]: of a tile: parts that it has, first row in the call, its place in the sequence's rows, how many
  int32_t* status;
};

// Sequences of up to so many rows (new tokens x query heads of a group) are the form for few rows', which reads the cache once for every 16 of them but
// shares it out evenly over the SMs.  us of one sequence of 8192 tokens, 8 heads of 128, few / many: 36 rows 24.2 / 35.7, 64 rows 26.8 / 37.4, 128
// rows 36.4 / 43.4, 256 rows 56.9 / 49.0.  Sixteen sequences of 2000 tokens, which fill the SMs with tiles: 20 rows 39.0 / 38.3, 32 rows 40.1 / 38.3, 64 rows
// 67.7 / 38.7, 128 rows 119.5 / 39.7; eight of 20000, a query head to a head: 20 rows 118 / 171.
static inline int lq_attn_few(int sequences, int heads, int sms) { return 2ll * sequences * heads < sms ? 128 : 32; }

lq_status lq_attn_tile_launch(const lq_kvcache* C, LqAttnParams p, cudaStream_t st);

#ifdef __CUDACC__
// A row's reference m is one of its products, as it is: the weight of product s is 2^((s - m) c).  Where c m is within LQ_ATTN_FAR, c s - c m in one
// fused operation is that, but for the rounding of c m, at most 2^-15, which all weights below one m share.  Farther out half a step of c m is
// added to every exponent, 16 and more from 2^28 on, and weights are infinite or nothing: there m is taken off the products first.
//
// m is followed lazily, once a product is LQ_ATTN_GROWTH above it, and weights are all LQ_ATTN_LIFT powers of two larger than that: up to 2^15 as
// halves (which go to 65504), so that small ones keep their 11 bits down to 2^-21 of m's, and are rounded by 2^-32 of it below.  (Without the lift
// 100000 tokens that one outweighs by e^17 each were rounded up by half of what they weigh, by e^17.5 to nothing, while the sum had them.)
constexpr float LQ_ATTN_FAR = 1024.f, LQ_ATTN_GROWTH = 8.f, LQ_ATTN_LIFT = 7.f;
__device__ __forceinline__ bool lq_attn_far(float m, float scale) { return m > -INFINITY && fabsf(m * scale) > LQ_ATTN_FAR; }
// what c s is moved by, once m has been taken off s where it is far out; a row that has seen nothing yet has no m
__device__ __forceinline__ float lq_attn_move(float m, float scale) {
  return m > -INFINITY && !lq_attn_far(m, scale) ? LQ_ATTN_LIFT - m * scale : LQ_ATTN_LIFT;
}
// c (its sign is the queries'); of a scale of zero: all weights are one, and what is not seen stays -inf
__device__ __forceinline__ float lq_attn_scale(const LqAttnParams& p) { return fmaxf(fabsf(p.scale), 1e-30f); }
// Tokens that any of the rows at places lo .. hi of a sequence may see, as blocks of 32: the first `sink` ones and those from `from` to `to` - 1;
// the b-th of them, and how many.
struct LqSeen {
  int sink, from, to;
  __device__ __forceinline__ int count() const { return sink + to - from; }
  __device__ __forceinline__ int block(int b) const { return b < sink ? b : b - sink + from; }
};
__device__ __forceinline__ LqSeen lq_seen(const LqAttnParams& p, int lo, int hi, int len) {
  const auto blocks = [](int tokens) { return (int)(((uint32_t)tokens + LQ_KV_BLOCK - 1) / LQ_KV_BLOCK); };
  LqSeen s{0, 0, blocks(len)};
  if (p.causal) {
    s.to = hi / LQ_KV_BLOCK + 1;
    if (p.window > 0 && lo >= p.window) {
      s.from = (lo - p.window + 1) / LQ_KV_BLOCK;
      s.sink = min(s.from, blocks(min(p.sinks, len)));
    }
  }
  return s;
}
// whether the row at place `at` sees token t
__device__ __forceinline__ bool lq_sees(const LqAttnParams& p, int at, int t, int len) {
  if (!p.causal) return t < len;
  return t <= at && (p.window == 0 || t > at - p.window || t < p.sinks);
}
// whether all rows at places lo .. hi see all tokens t0 .. t1
__device__ __forceinline__ bool lq_all_seen(const LqAttnParams& p, int lo, int hi, int t0, int t1, int len) {
  if (!p.causal) return t1 < len;
  return t1 <= lo && (p.window == 0 || t0 > hi - p.window || t1 < p.sinks);
}
// whether this launch takes a sequence, and whether it can be taken at all
__device__ __forceinline__ bool lq_attn_takes(const LqAttnParams& p, const LqSeq& q, bool tell) {
  if (q.n == 0) return false;
  const long long rows = (long long)q.n * p.group;
  if (rows < p.few || rows >= p.many) return false;
  if (!lq_seq_fits(p.b, q) || (p.causal && q.len < q.n)) {
    if (tell) lq_kv_refuse(p.status);
    return false;
  }
  return true;
}
#endif
