// A paged cache of keys and values in 8 bits: quantised as it is written, and read back.
//
//   a block of 32 tokens of a head has one step 2^e for its keys and one for its values, e the smallest integer in [-20, 9] with
//   127 * 2^e >= the largest magnitude that was written to it;   code c = rint(x / 2^e) in [-127, 127]
//
// Tokens that come to a block that has some already may need a larger e'; the codes that are there become rint(c / 2^(e' - e)).  Powers of two make
// both divisions exact, and every value c 2^e is a half (of 11 bits: c has 7).
//
// Both kernels are the memory's: rows in and codes out, or the other way round, once.  Two warps have the keys of a head's block and two its values; rows go
// through registers 16 bytes a lane and records through shared memory, where they change order (straight from rows to a record's places: 133 us
// for 79).  B200: 32768 rows of 8 heads of 128 written in 46 us and read in 34, 0.69 and 0.91 of the measured copy rate of their bytes (written:
// the blocks' two meetings, and registers for 28 warps an SM); single tokens of 32 sequences, written and read, 6.1 us, latency.
#include <math.h>

#include <algorithm>
#include <new>

#include "lq_device.cuh"
#include "lq_heads_places.h"
#include "lq_kvcache.h"

using namespace lqdev;

namespace {

constexpr int THREADS = 128;             // two warps for the keys of a block of tokens, two for its values

struct RowsParams {
  LqBatch b;
  uint8_t* records;
  void *k, *v;
  long long seq[2], row[2], head[2];     // strides in elements
  int D, Dp, tile;                       // append: tile: rows that a thread block looks through
  const int32_t* begin;
  int most, blocks;                      // read: most tokens of a sequence, blocks that they can touch
  int32_t* status;
};

__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }
// smallest e in range with 127 * 2^e >= top
__device__ __forceinline__ int exponent_of(float top) {
  const uint32_t bits = __float_as_uint(top);
  // top = (1 + m) 2^x: 127 * 2^(x - 6) = (1 + 63 / 64) 2^x
  const int x = (int)(bits >> 23) - 127, e = x - 6 + ((bits & 0x7FFFFF) > (63u << 17));
  return max(LQ_KV_E_MIN, min(LQ_KV_E_MAX, e));
}
// rint(c / 2^k) of a byte c + 128
__device__ __forceinline__ uint32_t shrink(uint32_t u, float inv) { return (uint32_t)(__float2int_rn((float)((int)u - 128) * inv) + 128); }

// Eight neighbouring entries of a token, as they lie in memory: their largest magnitude, and their codes as bytes c + 128, four to a word.
// FMA with a constant whose last place is one rounds to whole numbers, to even in the middle, and leaves the byte as the lowest of the sum.
template <typename T> struct Raw8;
template <> struct Raw8<__half> {
  uint4 v;
  __device__ __forceinline__ static Raw8 load(const __half* p) { return {*reinterpret_cast<const uint4*>(p)}; }
  __device__ __forceinline__ static Raw8 zero() { return {make_uint4(0, 0, 0, 0)}; }
  __device__ __forceinline__ float top(float m) const {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    __half2 a = __habs2(*reinterpret_cast<const __half2*>(&w[0]));
#pragma unroll
    for (int i = 1; i < 4; ++i) a = __hmax2(a, __habs2(*reinterpret_cast<const __half2*>(&w[i])));
    return fmaxf(m, __half2float(__hmax(__low2half(a), __high2half(a))));
  }
  __device__ __forceinline__ uint2 codes(int e) const {
    // 2^-e is a half down to e = -15; below that in two steps, both exact
    const __half2 first = __float2half2_rn(e < -15 ? 32.f : 1.f), rest = __float2half2_rn(pow2(e < -15 ? -e - 5 : -e)), place = __float2half2_rn(1664.f);
    const __half2 most = __float2half2_rn(65024.f), least = __float2half2_rn(-65024.f);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t c[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      __half2 x = *reinterpret_cast<const __half2*>(&w[i]);
      if (e == LQ_KV_E_MAX) x = __hmax2(least, __hmin2(most, x));
      x = __hfma2(__hmul2(x, first), rest, place);
      c[i] = *reinterpret_cast<const uint32_t*>(&x);
    }
    return make_uint2(__byte_perm(c[0], c[1], 0x6420), __byte_perm(c[2], c[3], 0x6420));
  }
};
template <> struct Raw8<float> {
  float4 a, b;
  __device__ __forceinline__ static Raw8 load(const float* p) { return {reinterpret_cast<const float4*>(p)[0], reinterpret_cast<const float4*>(p)[1]}; }
  __device__ __forceinline__ static Raw8 zero() { return {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)}; }
  __device__ __forceinline__ float top(float m) const {
    m = fmaxf(fmaxf(m, fmaxf(fabsf(a.x), fabsf(a.y))), fmaxf(fabsf(a.z), fabsf(a.w)));
    return fmaxf(fmaxf(m, fmaxf(fabsf(b.x), fabsf(b.y))), fmaxf(fabsf(b.z), fabsf(b.w)));
  }
  __device__ __forceinline__ uint2 codes(int e) const {
    const float inv = pow2(-e), place = 12582912.f + 128.f;
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    uint32_t c[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      float y = x[i];
      if (e == LQ_KV_E_MAX) y = fminf(fmaxf(y, -65024.f), 65024.f);
      c[i] = __float_as_uint(fmaf(y, inv, place));
    }
    return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
  }
};

// The sequence that row r belongs to, the last one that begins at or before it and has rows, and its rows and tokens; found by the warp together, in
// one trip to memory for up to 32 sequences (appends to ones of a single token, written and read, 6.7 -> 6.5 us).
__device__ __forceinline__ int sequence_of(const LqBatch& b, int r, int lane, LqSeq& q) {
  if (!b.row_start) {
    const int s = r / b.each;
    q = lq_seq(b, s);
    return s;
  }
  int lo = 0, n = b.sequences;           // the answer is in [lo, lo + n)
  while (n > 32) {
    const int step = (n + 31) / 32, at = lo + lane * step;
    const bool before = at < lo + n && b.row_start[at] <= r;
    const int last = 31 - __clz(__ballot_sync(0xffffffffu, before) | 1);
    lo += last * step;
    n = min(step, n - last * step);
  }
  LqSeq mine = {0, 0, 0};
  bool before = false;
  if (lane < n) {
    mine = lq_seq(b, lo + lane);
    before = b.row_start[lo + lane] <= r;
  }
  const int last = 31 - __clz(__ballot_sync(0xffffffffu, before) | 1);
  q.row = __shfl_sync(0xffffffffu, mine.row, last);
  q.n = __shfl_sync(0xffffffffu, mine.n, last);
  q.len = __shfl_sync(0xffffffffu, mine.len, last);
  return lo + last;
}

// A side of a record in shared memory, between rows and the order that it is kept in.  A thread turns units of four neighbouring tokens (a
// quad, of eight) times eight neighbouring entries (a chunk), so that rows are read and written 16 bytes a lane, whole rows by neighbouring
// lanes, and the record eight bytes at a time.  Lanes: bit 0 the upper half of a quad's number, the others the chunk; the warp the rest of the
// quad's number.  Records' 16-byte pieces change places within groups of eight, so that these eight bytes meet in no bank.
template <bool KEYS>
__device__ __forceinline__ int piece(int n) {
  const int g = n >> 5;
  return n ^ (KEYS ? (g & 1) | (g & 2) << 1 : (g & 3) | (n >> 2 & 4));
}
struct Unit {
  int upper, quad, chunk;                // the quad is 4 * upper + quad
  __device__ __forceinline__ int token(int x) const { return 16 * upper + 4 * quad + x; }
  // the i-th eight bytes: keys: entries 4 (i / 2) .. of the chunk, tokens 2 (i % 2), 2 (i % 2) + 1; values: entries 2 i, 2 i + 1, all tokens
  template <bool KEYS>
  __device__ __forceinline__ int at(int i) const {
    const int n = KEYS ? (chunk >> 1) * 32 + (2 * quad + (i & 1)) * 4 + (chunk & 1) * 2 + (i >> 1) : (chunk >> 1) * 32 + ((chunk & 1) * 4 + i) * 4 + quad;
    return piece<KEYS>(n) * 16 + upper * 8;
  }
};
// keys' and values' warps meet, each in code of their own
__device__ __forceinline__ void meet() { asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory"); }
__device__ __forceinline__ uint2 lds_v2(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ void sts_v2(uint32_t a, const uint2& v) { asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(v.x), "r"(v.y) : "memory"); }

// One block, keys or values, that has no tokens yet, two warps: tokens 0 .. n - 1 are rows of `in`, the others zeros.
template <typename T, bool KEYS, int CHUNKS>
__device__ __forceinline__ void fill_block(const RowsParams& p, int block, int slot, int page, int head, const T* in, long long row, int n, uint32_t image, float* tops) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5 & 1, D = p.D, groups = (D + 15) / 16;
  const long long found = lq_kv_at(p.b, block, slot, page);
  if (found < 0) {
    if (threadIdx.x == 0) lq_kv_refuse(p.status);
    return;
  }
  uint8_t* record = p.records + (found + head) * p.b.record;
  Raw8<T> raw[CHUNKS][2][4];
  float top = 0.f;
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const Unit u{lane & 1, 2 * q + warp, (lane >> 1) + 16 * c};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        raw[c][q][x] = Raw8<T>::zero();
        if (8 * u.chunk < D && u.token(x) < n) raw[c][q][x] = Raw8<T>::load(in + u.token(x) * row + 8 * u.chunk);
      }
    }
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int x = 0; x < 4; ++x) top = raw[c][q][x].top(top);
#pragma unroll
  for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  if (lane == 0) tops[threadIdx.x >> 5] = top;
  meet();
  const int e = exponent_of(fmaxf(tops[KEYS ? 0 : 2], tops[KEYS ? 1 : 3]));
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const Unit u{lane & 1, 2 * q + warp, (lane >> 1) + 16 * c};
      if (u.chunk >= 2 * groups) continue;
      uint2 w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) w[x] = raw[c][q][x].codes(e);
      if constexpr (KEYS) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          sts_v2(image + u.at<true>(i), make_uint2(w[2 * i].x, w[2 * i + 1].x));
          sts_v2(image + u.at<true>(2 + i), make_uint2(w[2 * i].y, w[2 * i + 1].y));
        }
      } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {                      // four tokens' bytes of four entries, rows for columns
          const uint32_t t0 = i ? w[0].y : w[0].x, t1 = i ? w[1].y : w[1].x, t2 = i ? w[2].y : w[2].x, t3 = i ? w[3].y : w[3].x;
          const uint32_t a = __byte_perm(t0, t1, 0x5140), b = __byte_perm(t2, t3, 0x5140), c2 = __byte_perm(t0, t1, 0x7362), d2 = __byte_perm(t2, t3, 0x7362);
          sts_v2(image + u.at<false>(2 * i), make_uint2(__byte_perm(a, b, 0x5410), __byte_perm(a, b, 0x7632)));
          sts_v2(image + u.at<false>(2 * i + 1), make_uint2(__byte_perm(c2, d2, 0x5410), __byte_perm(c2, d2, 0x7632)));
        }
      }
    }
  meet();
  uint4* to = reinterpret_cast<uint4*>(record + LQ_KV_HEAD + (KEYS ? 0 : lq_kv_side_bytes(p.Dp)));
  for (int i = threadIdx.x & 63; i < 32 * groups; i += 64) to[i] = lds_v4(image + piece<KEYS>(i) * 16);
  if ((threadIdx.x & 63) == 0) reinterpret_cast<int8_t*>(record)[KEYS ? 0 : 1] = (int8_t)e;
}

// One block, keys or values, one warp: tokens t0 .. t1 - 1 of it are new, rows of `in` from that of t0 on; those before t0 (there are some) are there
// already.
template <typename T, bool KEYS>
__device__ __forceinline__ void add_to_block(uint8_t* record, const T* in, long long row, int t0, int t1, int D, int Dp) {
  const int lane = threadIdx.x & 31, chunks = D / 8, n = t1 - t0;
  int8_t* exps = reinterpret_cast<int8_t*>(record) + (KEYS ? 0 : 1);
  const int was = max(LQ_KV_E_MIN, min(LQ_KV_E_MAX, (int)*reinterpret_cast<volatile int8_t*>(exps)));
  float top = 0.f;
  for (int i = lane; i < n * chunks; i += 32) {
    const int r = i / chunks, c = i - r * chunks;
    top = Raw8<T>::load(in + r * row + 8 * c).top(top);
  }
#pragma unroll
  for (int d = 16; d > 0; d /= 2) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
  const int e = max(exponent_of(top), was);
  uint8_t* side = record + LQ_KV_HEAD + (KEYS ? 0 : lq_kv_side_bytes(Dp));
  if (e > was) {                                           // what is there is rounded to the larger step
    const float less = pow2(was - e);
    const int c8 = lane >> 2, t = lane & 3;
    for (int g = 0; 16 * g < D; ++g) {
      uint4* at = reinterpret_cast<uint4*>(side + 512 * g + 16 * lane);
      const uint4 v = *at;
      uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (KEYS ? lq_kv_token(c8, i) >= t0 : 16 * (i >> 1) + 4 * t >= t0) continue;
        w[i] = shrink(w[i] & 0xFF, less) | shrink((w[i] >> 8) & 0xFF, less) << 8 | shrink((w[i] >> 16) & 0xFF, less) << 16 | shrink(w[i] >> 24, less) << 24;
      }
      *at = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (lane == 0) *exps = (int8_t)e;
    __syncwarp();
  }
  for (int i = lane; i < n * chunks; i += 32) {            // (bytes of other tokens in the same words stay)
    const int r = i / chunks, c = i - r * chunks, token = t0 + r, quad = token >> 2 & 3, s = token >> 4;
    const uint2 w = Raw8<T>::load(in + r * row + 8 * c).codes(e);
    if constexpr (KEYS) {
      const int column = 2 * quad + (token >> 1 & 1), word = 2 * s + (token & 1);
      uint32_t* at = reinterpret_cast<uint32_t*>(side + 512 * (c >> 1) + (column * 4 + (c & 1) * 2) * 16 + word * 4);
      at[0] = w.x;
      at[4] = w.y;
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        side[512 * (c >> 1) + (((c & 1) * 4 + (k >> 1)) * 4 + quad) * 16 + s * 8 + (k & 1) * 4 + (token & 3)] = (uint8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
    }
  }
}

// A thread block takes a head in the blocks of tokens that begin within its tile of rows: with a sequence's first new row, or with a token that
// is the first of its block.
template <typename T, int CHUNKS>
__global__ void __launch_bounds__(THREADS) lq_kv_append_kernel(const __grid_constant__ RowsParams p) {
  __shared__ __align__(16) uint8_t images[2][16 * CHUNKS * 256];
  __shared__ float tops[THREADS / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, side = warp >> 1;
  grid_launch_dependents();
  grid_dependency_wait();
  const int head = blockIdx.x % p.b.heads;
  int r = (int)(blockIdx.x / p.b.heads) * p.tile;
  const int end = min(p.b.rows - r, p.tile) + r;
  const T* in = reinterpret_cast<const T*>(side ? p.v : p.k) + head * p.head[side];
  LqSeq q;
  int s = sequence_of(p.b, r, lane, q);
  for (bool known = true; r < end && s < p.b.sequences; known = false) {
    if (!known) q = lq_seq(p.b, s);
    if (r < q.row || q.n == 0 || r >= q.row + q.n) {       // rows of no sequence lie in front (then r moves on), or the next sequence has it
      if (r < q.row) r = q.row;
      else ++s;
      continue;
    }
    if (!lq_seq_fits(p.b, q) || q.len < q.n) {
      if (threadIdx.x == 0) lq_kv_refuse(p.status);
      r = q.row + q.n;
      continue;
    }
    const int at = q.len - q.n + (r - q.row), t0 = at % LQ_KV_BLOCK, t1 = min(LQ_KV_BLOCK, t0 + (q.row + q.n - r));
    if (r == q.row || t0 == 0) {
      const int block = at / LQ_KV_BLOCK, slot = lq_kv_slot(p.b, block), page = p.b.pages[(long long)s * p.b.page_stride + slot];
      const T* rows = in + r * p.row[side];
      if (t0 == 0) {
        __syncthreads();                                   // (the images of the block before are read)
        if (side == 0) fill_block<T, true, CHUNKS>(p, block, slot, page, head, rows, p.row[0], t1, smem_u32(images[0]), tops);
        else fill_block<T, false, CHUNKS>(p, block, slot, page, head, rows, p.row[1], t1, smem_u32(images[1]), tops);
      } else {
        const long long found = lq_kv_at(p.b, block, slot, page);
        if (found < 0) {
          if (threadIdx.x == 0) lq_kv_refuse(p.status);
        } else {
          uint8_t* record = p.records + (found + head) * p.b.record;
          if (warp == 0) add_to_block<T, true>(record, rows, p.row[0], t0, t1, p.D, p.Dp);
          else if (warp == 2) add_to_block<T, false>(record, rows, p.row[1], t0, t1, p.D, p.Dp);
        }
      }
    }
    r += t1 - t0;
  }
}

// Four neighbouring values, as halves times 16 (they were opened as 2^-4 of themselves)
__device__ __forceinline__ uint32_t whole(uint32_t v) {
  const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&v), __float2half2_rn(16.f));
  return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ void store8(__half* p, const uint32_t (&w)[4]) { *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
__device__ __forceinline__ void store8(float* p, const uint32_t (&w)[4]) {
  float2 f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
  reinterpret_cast<float4*>(p)[0] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
  reinterpret_cast<float4*>(p)[1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
}
template <typename T, bool KEYS, int CHUNKS>
__device__ __forceinline__ void open_block(const uint8_t* record, T* out, long long row, int from, int to, int D, int Dp, uint32_t image) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5 & 1, groups = (D + 15) / 16;
  const uint4* units = reinterpret_cast<const uint4*>(record + LQ_KV_HEAD + (KEYS ? 0 : lq_kv_side_bytes(Dp)));
  const uint32_t high = lq_kv_high(reinterpret_cast<const int8_t*>(record)[KEYS ? 0 : 1]);
  const __half2 less = lq_kv_less(high);
#pragma unroll
  for (int i = 0; i < 4 * CHUNKS; ++i) {
    const int n = (threadIdx.x & 63) + 64 * i;
    if (n < 32 * groups) sts_v4(image + piece<KEYS>(n) * 16, units[n]);
  }
  meet();
#pragma unroll
  for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const Unit u{lane & 1, 2 * q + warp, (lane >> 1) + 16 * c};
      if (8 * u.chunk >= D) continue;
      uint32_t w[4][4];                                    // [token][pair of entries]
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint2 v = lds_v2(image + u.at<KEYS>(i));
        if constexpr (KEYS) {
          const int x = 2 * (i & 1), d = 2 * (i >> 1);
          w[x][d] = lq_kv_open<0x4140>(v.x, high, less); w[x][d + 1] = lq_kv_open<0x4342>(v.x, high, less);
          w[x + 1][d] = lq_kv_open<0x4140>(v.y, high, less); w[x + 1][d + 1] = lq_kv_open<0x4342>(v.y, high, less);
        } else {
          const uint32_t a = __byte_perm(v.x, v.y, 0x5140), b = __byte_perm(v.x, v.y, 0x7362);
          w[0][i] = lq_kv_open<0x4140>(a, high, less); w[1][i] = lq_kv_open<0x4342>(a, high, less);
          w[2][i] = lq_kv_open<0x4140>(b, high, less); w[3][i] = lq_kv_open<0x4342>(b, high, less);
        }
      }
#pragma unroll
      for (int x = 0; x < 4; ++x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[x][i] = whole(w[x][i]);
        const int token = u.token(x);
        if (token >= from && token < to) store8(out + token * row + 8 * u.chunk, w[x]);
      }
    }
}

// A thread block takes a head in one block of tokens.
template <typename T, int CHUNKS>
__global__ void __launch_bounds__(THREADS) lq_kv_read_kernel(const __grid_constant__ RowsParams p) {
  __shared__ __align__(16) uint8_t images[2][16 * CHUNKS * 256];
  const int side = threadIdx.x >> 6, head = blockIdx.x % p.b.heads;
  grid_launch_dependents();
  grid_dependency_wait();
  const int rest = blockIdx.x / p.b.heads, s = rest / p.blocks, i = rest - s * p.blocks;
  LqSeq q;
  q.len = p.b.length[s];
  const int begin = p.begin ? p.begin[s] : 0;
  if (!lq_seq_fits(p.b, q) || begin < 0) {
    if (threadIdx.x == 0) lq_kv_refuse(p.status);
    return;
  }
  const long long block = (long long)begin / LQ_KV_BLOCK + i;
  const int end = (int)min((long long)q.len, (long long)begin + p.most);
  if (block * LQ_KV_BLOCK >= end) return;
  const long long at = lq_kv_at(p.b, s, (int)block);
  if (at < 0) {
    if (threadIdx.x == 0) lq_kv_refuse(p.status);
    return;
  }
  const uint8_t* record = p.records + (at + head) * p.b.record;
  const int first = (int)(block * LQ_KV_BLOCK), from = max(0, begin - first), to = min(LQ_KV_BLOCK, end - first);
  T* out = reinterpret_cast<T*>(side ? p.v : p.k) + s * p.seq[side] + head * p.head[side] + ((long long)first - begin) * p.row[side];
  if (side == 0) open_block<T, true, CHUNKS>(record, out, p.row[0], p.k ? from : LQ_KV_BLOCK, to, p.D, p.Dp, smem_u32(images[0]));
  else open_block<T, false, CHUNKS>(record, out, p.row[1], p.v ? from : LQ_KV_BLOCK, to, p.D, p.Dp, smem_u32(images[1]));
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

LqPlaces lq_batch_meets(const LqBatch& b, const int32_t* more, int entries, const LqRuns& out) {
  const auto line = [](const int32_t* at, int64_t n) { return LqRuns{(uintptr_t)at, {0, 0, 0}, {1, 1, 1}, 4 * n}; };
  const LqRuns arrays[3] = {line(b.length, b.sequences), line(b.pages, (int64_t)b.sequences * b.page_stride), line(more, entries)};
  for (const LqRuns& a : arrays) {
    const LqPlaces c = a.at ? lq_runs_meet(out, a) : LQ_APART;
    if (c != LQ_APART) return c;
  }
  return LQ_APART;
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
      lq_note_cuda(cudaMalloc((void**)&C->d_count, C->sms * sizeof(int))) != cudaSuccess ||
      (Dp <= 128 && (lq_note_cuda(cudaMalloc((void**)&C->d_tile_part, (size_t)C->sms * 256 * (Dp + 2) * sizeof(float))) != cudaSuccess ||
                     lq_note_cuda(cudaMalloc((void**)&C->d_tile_meta, C->sms * sizeof(int4))) != cudaSuccess))) {
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
  cudaFree(C->d_records); cudaFree(C->d_part); cudaFree(C->d_count); cudaFree(C->d_tile_part); cudaFree(C->d_tile_meta);
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
  // Rows a thread block looks through: 32, as many as a block of tokens has, once that gives every SM eight; with fewer rows fewer, so that
  // single tokens of different sequences are not one's.
  p.tile = (int)std::max(1ll, std::min(32ll, (long long)C->heads * p.b.rows / (8ll * C->sms)));
  const long long blocks = C->heads * (1ll + (p.b.rows - 1) / p.tile);
  if (blocks > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  const auto launch = [&](auto* kernel) { return lq_launch(kernel, (int)blocks, THREADS, 0, (cudaStream_t)stream, p); };
  const cudaError_t e = dt == LQ_OUT_F16 ? (C->D <= 128 ? launch(lq_kv_append_kernel<__half, 1>) : launch(lq_kv_append_kernel<__half, 2>))
                                         : (C->D <= 128 ? launch(lq_kv_append_kernel<float, 1>) : launch(lq_kv_append_kernel<float, 2>));
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
  // no two entries of the outputs on one place, and none on the arrays
  LqRuns out[2];
  int n = 0;
  for (int i = 0; i < 2; ++i)
    if (i == 0 ? p.k : p.v) {
      const int64_t esz = dt == LQ_OUT_F32 ? 4 : 2;
      out[n++] = LqRuns{(uintptr_t)(i == 0 ? p.k : p.v), {p.seq[i] * esz, p.row[i] * esz, p.head[i] * esz}, {p.b.sequences, p.most, C->heads}, C->D * esz};
    }
  const auto status = [](LqPlaces c) { return c == LQ_APART ? LQ_OK : c == LQ_SHARED ? LQ_ERR_INVALID_ARG : LQ_ERR_UNSUPPORTED; };
  for (int i = 0; i < n; ++i)
    if ((s = status(lq_runs_collide(out[i]))) != LQ_OK || (s = status(lq_batch_meets(p.b, begin, p.b.sequences, out[i]))) != LQ_OK) return s;
  if (n == 2 && (s = status(lq_runs_meet(out[0], out[1]))) != LQ_OK) return s;
  LqDeviceGuard guard(C->device);
  if (!guard.ok) return LQ_ERR_CUDA;
  p.records = lq_kv_layer(C, layer);
  p.D = C->D; p.Dp = C->Dp;
  p.status = lq_device_status_ptr(C->device);
  const long long blocks = (long long)C->heads * p.b.sequences * p.blocks;
  if (blocks > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  const auto launch = [&](auto* kernel) { return lq_launch(kernel, (int)blocks, THREADS, 0, (cudaStream_t)stream, p); };
  const cudaError_t e = dt == LQ_OUT_F16 ? (C->D <= 128 ? launch(lq_kv_read_kernel<__half, 1>) : launch(lq_kv_read_kernel<__half, 2>))
                                         : (C->D <= 128 ? launch(lq_kv_read_kernel<float, 1>) : launch(lq_kv_read_kernel<float, 2>));
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
