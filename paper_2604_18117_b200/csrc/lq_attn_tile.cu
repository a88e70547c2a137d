// Attention over the cache, the form for many rows of heads of up to 128 entries: tiles of 256 rows (new tokens x query heads of a group) on
// tcgen05.
//
//   S = Q K^T,   P = 2^(S c - m c),   O += P V,   l += P 1        over 128 tokens (four records) at a time, m a maximum of the row so far
//
// What bounds it is the tensor cores and what feeds them.  Seven warps open the records to halves in shared memory (two buffers of K and V, in
// swizzled rows, where no two lanes of a store meet in a bank); one thread issues the products; two groups of four warps have 128 rows each, a
// row a thread, and take turns with the tensor cores: while one forms P of its rows, the products of the other run, and O's product follows P
// 64 tokens at a time.  S and O stay in tensor memory.  P, as halves, takes the place of S and is the second product's A operand from
// there.  O is only scaled when a row's maximum has grown by 8 or more (in powers of two) since it was last: until then weights are that much
// larger, which halves and sums hold as well (lq_attn.h), and the last division takes care of it.
//
// B200, us of passes back to back in graphs: 4096 tokens behind 4096, 32 heads of 128 on 8 414 at 1.83 GHz, which the power limit leaves (996 TFLOP/s of
// visible pairs, 0.59 of the measured burst rate of a GEMM, 0.71 of the sustained one; the first ten passes after a pause 396 each); two images of 4096
// tokens, 16 heads of 72 242 at 1.965 GHz (119 of them are the powers' at 16 a clock).  A tile of 128 tokens takes some 4000 clocks where the tensor
// cores need 2048: the chain S -> weights -> O of either half and its hand-overs.  What follows is of ten passes after a pause, side by side in the builds
// of their time, and good for comparison alone.  With P in four pieces and no powers it took 0.99 of 415,
// without maxima, sums and powers 0.96, without opening the records 0.95, with an eighth of S's product 0.84, with none of all that still 0.69.  So what
// counts is how often there is something to wait for: P in one, two or four pieces 391, 387 and 415.  Timed and not kept: two threads a row (16 warps:
// 441 for 430), the first weights by the last maximum while the new one is found (437), an eighth to a half of the powers by polynomials (431 to 502
// for 445), S of 64 tokens twice so that the next one's product runs under a weighing (493, and 401 with a thread for the products of each half, but
// images 257), issuing by lane 0 instead of an elected one (496 for 415); of the first form, which took 548, core matrices 16 and 32 bytes off
// boundaries of 128, whose stores met in no bank (588).
#include <math.h>

#include <algorithm>

#include "lq_attn.h"
#include "lq_device.cuh"

using namespace lqdev;

namespace {

constexpr int TILE = 128, KV = 128, PIECES = 2, PIECE = KV / PIECES, SOFT_WARPS = 8, OPEN_WARPS = 7, MMA_WARP = SOFT_WARPS + OPEN_WARPS, THREADS = 32 * (MMA_WARP + 1);
// Registers of a thread: as the block is launched (the kernel's bound, and what ptxas reports), and of the first kind and the others after setmaxnreg,
// which takes from what the block was launched with and would wait for ever for more (every instance's own count is checked in lq_attn_tile_prepare).
constexpr int LAUNCH_REGS = 128, SOFT_REGS = 176, LEAN_REGS = 80;
static_assert(SOFT_WARPS * SOFT_REGS + (OPEN_WARPS + 1) * LEAN_REGS <= THREADS / 32 * LAUNCH_REGS && THREADS % 128 == 0 && THREADS * LAUNCH_REGS <= 65536, "");
constexpr int TMEM_COLS = 512;
constexpr uint32_t COL_S = 0, COL_O = 256;                 // of the first 128 rows; the other's are 128 columns on
constexpr int MIN_TILES = 4;             // of 128 tokens a thread block takes at least where a tile of rows is shared out

// Operands are K-major rows of 128 bytes (64 halves), 128-byte swizzle; a wider K has panel after panel.  Q and K: rows are rows and tokens, 64
// entries a panel; V: rows are the head's entries, 64 tokens a panel.
__host__ __device__ constexpr int q_bytes(int Dp) { return (Dp + 63) / 64 * TILE * 128; }
__host__ __device__ constexpr int k_bytes(int Dp) { return (Dp + 63) / 64 * KV * 128; }
__host__ __device__ constexpr int v_bytes(int Dp) { return KV / 64 * Dp * 128; }
// the keys or the values of a record, behind its head, for every opening warp
__host__ __device__ constexpr int raw_bytes(int Dp) { return LQ_KV_HEAD + LQ_KV_BLOCK * Dp; }

// What a block works on.
struct Task {
  LqSeq q;
  LqSeen seen;
  int s, head, row0, rows;               // rows: of up to 256
  int first, tiles, parts;               // tiles of 128 tokens: from the first-th of the rows' on so many; parts: thread blocks that have some
};

struct Control {
  uint64_t raw[OPEN_WARPS], q_full[2], k_full[2], k_empty[2], v_full[2], v_empty[2], s_full[2], p_full[2][PIECES], o_full[2];
  uint32_t tmem;
  alignas(4) uint8_t missing[4][4];                 // of the last tiles: whether record i is no page's
  int abort_flag;
  int place[2];
  Task task;
  int prefix[THREADS / 32];
};

__device__ __forceinline__ void tmem_ld_32(uint32_t taddr, uint32_t (&v)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]),
        "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]),
        "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
      : "r"(taddr)
      : "memory");
}
// what has been loaded is used behind this place alone
__device__ __forceinline__ void settled(uint32_t (&v)[32]) {
  asm volatile(""
               : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                 "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]),
                 "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]),
                 "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]));
}
__device__ __forceinline__ void tmem_st_16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]),
      "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the same product with A in tensor memory: row r in lane r, two halves a column
__device__ __forceinline__ void tc_mma_ta(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// Waits until all lanes' loads have come that v is made of, and holds back what follows: a fence hangs on the lanes' vote, so the vote's outcome, and with it
// every lane's v, has to be there first.  (No lane has a v of zeros, whose codes would all be -128: the fence is not taken.)
__device__ __forceinline__ void arrived(uint32_t v) {
  if (__ballot_sync(0xffffffffu, v != 0) == 0) fence_proxy_async();
}
__device__ __forceinline__ void sts_v2(uint32_t a, uint32_t x, uint32_t y) { asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(a), "r"(x), "r"(y) : "memory"); }

// A record's keys as rows of 64 entries a panel, its 32 tokens from `to` on.  The lane's word i is 8 bytes of row lq_kv_token(c8, i); in a half of the
// warp's lanes these 8 bytes take all banks once.  then(): all lanes' loads have come (a copy that was asked for without that has overtaken some
// of them; a proxy fence there waits for the stores as well).
template <int NK, typename Then>
__device__ __forceinline__ void open_keys(uint32_t from, uint32_t to, uint32_t head, int lane, const Then& then) {
  constexpr int BATCH = (NK + 1) / 2;
  const int c8 = lane >> 2, t = lane & 3;
  const uint32_t high = lq_kv_high((int8_t)(head & 0xFF));
  const __half2 less = lq_kv_less(high);
  uint32_t at[4], any = head;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = lq_kv_token(c8, i);
    at[i] = to + row * 128 + (((t >> 1) ^ (row & 7)) * 16) + (t & 1) * 8;
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    uint4 u[BATCH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x)
      if (b * BATCH + x < NK) u[x] = lds_v4(from + 512 * (b * BATCH + x) + 16 * lane);
#pragma unroll
    for (int x = 0; x < BATCH; ++x)
      if (b * BATCH + x < NK) any |= u[x].w;
    if (b == 1) {
      arrived(any);
      then();
    }
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const int g = b * BATCH + x;
      if (g >= NK) continue;
      const uint32_t ww[4] = {u[x].x, u[x].y, u[x].z, u[x].w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        sts_v2((at[i] ^ (32 * (g & 3))) + g / 4 * KV * 128, lq_kv_open<0x4140>(ww[i], high, less), lq_kv_open<0x4342>(ww[i], high, less));
    }
  }
}
// Its values: rows are entries, 64 tokens a panel, of which the record has the lower or upper half.  Words 2 s + i are 8 bytes of row 16 g + 2 c8 + i.
template <int NK, typename Then>
__device__ __forceinline__ void open_values(uint32_t from, uint32_t to, uint32_t exponent, int upper, int lane, const Then& then) {
  constexpr int BATCH = (NK + 1) / 2;
  const int c8 = lane >> 2, t = lane & 3;
  const uint32_t high = lq_kv_high((int8_t)(exponent & 0xFF));
  const __half2 less = lq_kv_less(high);
  uint32_t at[4], any = exponent;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int chunk = 4 * upper + 2 * (i >> 1) + (t >> 1), row = 2 * c8 + (i & 1);
    at[i] = to + row * 128 + ((chunk ^ (row & 7)) * 16) + (t & 1) * 8;
  }
#pragma unroll
  for (int b = 0; b < 2; ++b) {
    uint4 u[BATCH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x)
      if (b * BATCH + x < NK) u[x] = lds_v4(from + 512 * (b * BATCH + x) + 16 * lane);
#pragma unroll
    for (int x = 0; x < BATCH; ++x)
      if (b * BATCH + x < NK) any |= u[x].w;
    if (b == 1) {
      arrived(any);
      then();
    }
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const int g = b * BATCH + x;
      if (g >= NK) continue;
      const uint32_t ww[4] = {u[x].x, u[x].y, u[x].z, u[x].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) sts_v2(at[i] + g * 2048, lq_kv_open<0x4140>(ww[i], high, less), lq_kv_open<0x4342>(ww[i], high, less));
    }
  }
}
// zeros in place of record w
__device__ __forceinline__ void zero_rows(uint32_t stage, int w, int side, int Dp, int lane) {
  if (side == 0) {
    for (int i = lane; i < (Dp + 63) / 64 * 256; i += 32) sts_v4(stage + i / 256 * KV * 128 + 32 * w * 128 + i % 256 * 16, make_uint4(0, 0, 0, 0));
  } else {
    for (int i = lane; i < Dp * 4; i += 32) {              // four of a row's eight 16-byte pieces
      const int row = i / 4, chunk = 4 * (w & 1) + i % 4;
      sts_v4(stage + w / 2 * Dp * 128 + row * 128 + ((chunk ^ (row & 7)) * 16), make_uint4(0, 0, 0, 0));
    }
  }
}

// Which of the 32 tokens from `first` on the row at place `at` sees.
__device__ __forceinline__ uint32_t below(int n) { return (uint32_t)((1ull << max(0, min(32, n))) - 1); }
__device__ __forceinline__ uint32_t seen_of(const LqAttnParams& p, int at, int first, int len) {
  const int end = p.causal ? at + 1 : len;
  uint32_t m = below(end - first);
  if (p.window > 0) m &= ~below(at - p.window + 1 - first) | below(p.sinks - first);
  return m;
}
// Of a tile's list of blocks the run that rows at places lo .. hi see as a whole (but for blocks of first tokens, which count as seen in part).
__device__ __forceinline__ int2 seen_whole(const LqAttnParams& p, const LqSeen& seen, int lo, int hi, int len) {
  if (!p.causal) return make_int2(0, len / LQ_KV_BLOCK);
  const int behind = (lo + 1) / LQ_KV_BLOCK - seen.from + seen.sink;
  if (p.window == 0) return make_int2(0, behind);
  const int first = max(0, hi - p.window + 1 + LQ_KV_BLOCK - 1) / LQ_KV_BLOCK;
  return make_int2(max(seen.sink, first - seen.from + seen.sink), behind);
}

template <int NK>
__global__ void __maxnreg__(LAUNCH_REGS) lq_attn_tile_kernel(const __grid_constant__ LqAttnParams p) {
  constexpr int DP = 16 * NK;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint8_t* sq = smem;                                      // [2]
  uint8_t* sk = sq + 2 * q_bytes(DP);                      // [2]
  uint8_t* sv = sk + 2 * k_bytes(DP);                      // [2]
  uint8_t* raw = sv + 2 * v_bytes(DP);                     // [OPEN_WARPS]
  Control& c = *reinterpret_cast<Control*>(raw + OPEN_WARPS * raw_bytes(DP));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&c.q_full[i]), 4);
      mbar_init(smem_u32(&c.k_full[i]), 4);
      mbar_init(smem_u32(&c.v_full[i]), 4);
      mbar_init(smem_u32(&c.k_empty[i]), 1);
      mbar_init(smem_u32(&c.v_empty[i]), 1);
      mbar_init(smem_u32(&c.s_full[i]), 1);
      for (int x = 0; x < PIECES; ++x) mbar_init(smem_u32(&c.p_full[i][x]), 4);
      mbar_init(smem_u32(&c.o_full[i]), 1);
    }
    for (int i = 0; i < OPEN_WARPS; ++i) mbar_init(smem_u32(&c.raw[i]), 1);
    c.abort_flag = 0;
    mbar_init_fence();
  }
  grid_dependency_wait();

  // the block's sequence and tile of rows: blocks of a tile's heads follow each other, a sequence's last tiles (which see most) come first
  Task k = {};
  // (the first p.whole tiles have a block each, the others p.splits)
  const int shared = (int)blockIdx.x - p.whole, part = shared < 0 ? 0 : shared % p.splits, place = shared < 0 ? (int)blockIdx.x : p.whole + shared / p.splits;
  k.head = place % p.b.heads;
  const int unit = place / p.b.heads;
  if (!p.b.row_start) {
    const int each = (int)(((long long)p.b.each * p.group + 2 * TILE - 1) / (2 * TILE)), back = unit / p.b.sequences;
    k.s = unit - back * p.b.sequences;
    k.row0 = (each - 1 - back) * 2 * TILE;
    k.q = lq_seq(p.b, k.s);
    if (!lq_attn_takes(p, k.q, place < p.b.heads * p.b.sequences)) k.s = -1;
  } else {
    const int chunk = (p.b.sequences + THREADS - 1) / THREADS;
    int sum = 0;
    for (int s = tid * chunk; s < min(p.b.sequences, (tid + 1) * chunk); ++s) {
      const LqSeq q = lq_seq(p.b, s);
      if (lq_attn_takes(p, q, blockIdx.x == 0)) sum += (int)(((long long)q.n * p.group + 2 * TILE - 1) / (2 * TILE));
    }
    int up = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xffffffffu, up, d);
      if (lane >= d) up += v;
    }
    if (lane == 31) c.prefix[warp] = up;
    if (tid == 0) c.place[0] = -1;
    __syncthreads();
    int base = up - sum;
    for (int i = 0; i < warp; ++i) base += c.prefix[i];
    if (unit >= base && unit < base + sum)                 // in this thread's sequences
      for (int s = tid * chunk; s < min(p.b.sequences, (tid + 1) * chunk); ++s) {
        const LqSeq q = lq_seq(p.b, s);
        if (!lq_attn_takes(p, q, false)) continue;
        const int tiles = (int)(((long long)q.n * p.group + 2 * TILE - 1) / (2 * TILE));
        if (unit < base + tiles) {
          c.place[0] = s;
          c.place[1] = (tiles - 1 - (unit - base)) * 2 * TILE;
          break;
        }
        base += tiles;
      }
    __syncthreads();
    k.s = c.place[0];
    k.row0 = c.place[1];
    if (k.s >= 0) k.q = lq_seq(p.b, k.s);
  }
  const int base = k.q.len - k.q.n;
  if (k.s >= 0) {
    k.rows = min(2 * TILE, k.q.n * p.group - k.row0);
    k.seen = lq_seen(p, base + k.row0 / p.group, base + (k.row0 + k.rows - 1) / p.group, k.q.len);
    const int all = (k.seen.count() + 3) / 4, each = shared < 0 ? max(1, all) : max(MIN_TILES, (all + p.splits - 1) / p.splits);
    k.parts = max(1, (all + each - 1) / each);
    k.first = part * each;
    k.tiles = max(0, min(each, all - k.first));
    if (part >= k.parts) k.rows = 0;                       // (nothing is left for this block)
  }
  if (shared >= 0 && p.splits > 1 && part == 0 && tid == 0) p.tile_meta[place - p.whole] = make_int4(k.parts, k.q.row, k.row0, k.rows);
  if (k.rows == 0) return;                                 // (a launch for a batch whose sequences may all have few rows costs little then)
  if (warp == MMA_WARP) tmem_alloc(smem_u32(&c.tmem), TMEM_COLS);
  if (tid == 0) c.task = k;                                // (for code that has no registers for it)
  __syncthreads();
  grid_launch_dependents();                                // (a kernel that starts early finds this block's tensor memory taken)
  const uint32_t tmem = *const_cast<volatile uint32_t*>(&c.tmem);
  const int halves = k.rows > TILE ? 2 : 1, tiles = k.tiles;
  bool good = true;
  const auto wait = [&](uint64_t& bar, int phase, int role) {
    // (without a call: the warps' registers are not those that the block was launched with)
    if (good) good = __all_sync(0xffffffffu, mbar_wait_inline(smem_u32(&bar), phase & 1, &c.abort_flag, p.status, role));
    return good;
  };

  if (warp < SOFT_WARPS) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(SOFT_REGS));
    const int half = warp / 4, row = (warp & 3) * 32 + lane;
    if (half < halves && k.rows > 0) {
      const volatile Task& task = c.task;
      // the row: of the sequence's rows, behind which the last one stands in
      const auto row_of = [&](int i, int& tok) {
        const int r = min(task.row0 + half * TILE + i, task.q.n * p.group - 1);
        tok = r / p.group;
        return task.head * p.group + (r - tok * p.group);  // the query head
      };
      int2 whole;
      {
        int lo, hi;
        row_of((warp & 3) * 32, lo);
        row_of((warp & 3) * 32 + 31, hi);
        whole = seen_whole(p, k.seen, base + lo, base + hi, k.q.len);
        whole.x -= 4 * k.first; whole.y -= 4 * k.first;    // of the block's tiles
      }
      // the row of Q, with the sign of the scale
      {
        int tok;
        const long long head = row_of(row, tok);
        const bool real = k.row0 + half * TILE + row < k.q.n * p.group;
        const uint4* from = reinterpret_cast<const uint4*>(p.q + (k.q.row + tok) * p.q_row + head * p.q_head);
        const uint32_t flip = p.scale < 0.f ? 0x80008000u : 0u;
        const uint32_t to = smem_u32(sq + half * q_bytes(DP)) + row * 128;
#pragma unroll
        for (int g = 0; g < DP / 8; ++g) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (real && 8 * g < p.D) {
            v = from[g];
            v.x ^= flip; v.y ^= flip; v.z ^= flip; v.w ^= flip;
          }
          sts_v4(to + g / 8 * TILE * 128 + (((g & 7) ^ (row & 7)) * 16), v);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&c.q_full[half]));
      }
      const float scale = lq_attn_scale(p);
      const uint32_t ts = tmem + ((uint32_t)(warp & 3) << 21) + COL_S + half * 128, to = ts + COL_O - COL_S;
      float m = -INFINITY, move = 0.f, l = 0.f;            // m: the row's reference
      bool far = false;                                    // (some of the warp's rows' are)
      for (int j = 0; j < tiles; ++j) {
        if (!wait(c.s_full[half], j, LQ_STAGE_DRAIN)) break;
        tc_fence_after();
        const uint32_t missing = *reinterpret_cast<volatile uint32_t*>(c.missing[j & 3]);
        uint32_t v[4][32];
#pragma unroll
        for (int i = 0; i < 4; ++i) tmem_ld_32(ts + 32 * i, v[i]);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 4; ++i) settled(v[i]);
        // Of 32 tokens the weights, as they go to tensor memory, and what they add to the sum (taken to one number when all are handed over)
        const float2 scale2 = make_float2(scale, scale);
        uint32_t w[16];
        float2 sum[2] = {};
        const auto weigh = [&](const uint32_t (&v)[32]) {
          const float2 move2 = make_float2(move, move);
#pragma unroll
          for (int x = 0; x < 32; x += 2) {
            float2 e = __ffma2_rn(make_float2(__uint_as_float(v[x]), __uint_as_float(v[x + 1])), scale2, move2);
            e.x = ex2(e.x); e.y = ex2(e.y);
            sum[x / 2 & 1] = __fadd2_rn(sum[x / 2 & 1], e);
            w[x / 2] = pack(e.x, e.y);
          }
        };
        // (most tiles are seen by all rows as a whole)
        const bool covered = missing != 0 || 4 * j < whole.x || 4 * j + 3 >= whole.y;
        if (covered) {
          int tok;
          row_of(row, tok);
          const LqSeen seen{task.seen.sink, task.seen.from, task.seen.to};
          const int len = task.q.len, at = len - task.q.n + tok;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int b = 4 * (task.first + j) + i;
            const uint32_t mask = b < seen.count() && !(missing >> (8 * i) & 1) ? seen_of(p, at, seen.block(b) * LQ_KV_BLOCK, len) : 0;
#pragma unroll
            for (int x = 0; x < 32; ++x)
              if (!(mask >> x & 1)) v[i][x] = 0xff800000u; // -inf
          }
        }
        float top;
        {
          float t[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int x = 0; x < 32; x += 2) t[x / 2 & 3] = fmaxf(fmaxf(t[x / 2 & 3], __uint_as_float(v[i][x])), __uint_as_float(v[i][x + 1]));
          top = fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3]));
        }
        const bool grow = (top - m) * scale > LQ_ATTN_GROWTH;      // (also of the first product that a row sees; not where both are -inf)
        if (__any_sync(0xffffffffu, grow || far)) {
          // (a row that has seen nothing yet has sums of zero; its factor is one)
          const float by = grow && m > -INFINITY ? ex2((m - top) * scale) : 1.f;
          if (grow) { l *= by; m = top; move = lq_attn_move(m, scale); }
          if (j > 0 && __any_sync(0xffffffffu, by != 1.f))
#pragma unroll 1
            for (int x = 0; x < DP; x += 16) {
              uint32_t u[16];
              tmem_ld_32x16(to + x, u);
              tmem_ld_wait();
#pragma unroll
              for (int y = 0; y < 16; ++y) u[y] = __float_as_uint(__uint_as_float(u[y]) * by);
              tmem_st_16(to + x, u);
            }
          far = __any_sync(0xffffffffu, lq_attn_far(m, scale));
          if (far) {
            const float off = lq_attn_far(m, scale) ? m : 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int x = 0; x < 32; ++x) v[i][x] = __float_as_uint(__uint_as_float(v[i][x]) - off);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          weigh(v[i]);
          tmem_st_16(ts + 16 * i, w);                      // (over columns of S, which has been read)
          if ((i + 1) % (PIECE / 32) != 0) continue;
          tmem_st_wait();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&c.p_full[half][i / (PIECE / 32)]));
        }
        l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      }
      if (tiles > 0 && wait(c.o_full[half], 0, LQ_STAGE_DRAIN)) tc_fence_after();
      if (task.parts > 1) {                                // for lq_attn_join_kernel
        float* out = p.tile_part + (long long)(blockIdx.x - p.whole) * (DP + 2) * (2 * TILE) + half * TILE + row;
        if (good)
#pragma unroll 1
          for (int x = 0; x < DP; x += 16) {
            uint32_t v[16];
            tmem_ld_32x16(to + x, v);
            tmem_ld_wait();
#pragma unroll
            for (int y = 0; y < 16; ++y) out[(x + y) * (2 * TILE)] = __uint_as_float(v[y]);
          }
        out[DP * (2 * TILE)] = m;
        out[(DP + 1) * (2 * TILE)] = l;
      } else {
        // values were opened as 2^-4 of themselves
        const float by = l > 0.f ? 16.f / l : 0.f;
        int tok;
        const long long head = row_of(row, tok);
        const bool real = task.row0 + half * TILE + row < task.q.n * p.group;
        __half* out = p.out + (task.q.row + tok) * p.out_row + head * p.out_head;
        if (good)
#pragma unroll 1
          for (int x = 0; x < DP; x += 16) {
            uint32_t v[16] = {};
            if (tiles > 0) {
              tmem_ld_32x16(to + x, v);
              tmem_ld_wait();
            }
            uint32_t w[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) w[y] = pack(__uint_as_float(v[2 * y]) * by, __uint_as_float(v[2 * y + 1]) * by);
            if (real && x < p.D) *reinterpret_cast<uint4*>(out + x) = make_uint4(w[0], w[1], w[2], w[3]);
            if (real && x + 8 < p.D) *reinterpret_cast<uint4*>(out + x + 8) = make_uint4(w[4], w[5], w[6], w[7]);
          }
      }
      tc_fence_before();
    }
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(LEAN_REGS));
    if (warp < MMA_WARP) {
      // A tile's eight jobs, the keys of its four records and then the values, go round the seven warps.  What a job opens, with the record's head,
      // is copied to the warp's own place in shared memory; that of its next job is asked for as soon as this has been loaded.
      const int ow = warp - SOFT_WARPS, count = tiles > 0 ? k.seen.count() : 0;
      const uint32_t place = smem_u32(raw + ow * raw_bytes(DP)), bar = smem_u32(&c.raw[ow]);
      // the record of job n, null: behind the last or no page's.  Its page is asked for a job before.
      int page = -1;
      const auto ask = [&](int n) {
        const int b = 4 * (k.first + (n >> 3)) + (n & 3);
        if (n < 8 * tiles && b < count) page = p.b.pages[(long long)k.s * p.b.page_stride + lq_kv_slot(p.b, k.seen.block(b))];
      };
      const auto find = [&](int n) -> const uint8_t* {
        const int b = 4 * (k.first + (n >> 3)) + (n & 3);
        if (n >= 8 * tiles || b >= count) return nullptr;
        const int block = k.seen.block(b);
        const long long x = lq_kv_at(p.b, block, lq_kv_slot(p.b, block), page);
        if (x < 0 && lane == 0) lq_kv_refuse(p.status);
        return x < 0 ? nullptr : p.records + (x + k.head) * p.b.record;
      };
      const auto fetch = [&](int n, const uint8_t* rec) {
        if (rec && lane == 0) {
          mbar_expect_tx(bar, LQ_KV_HEAD + LQ_KV_BLOCK * DP);
          if ((n & 4) == 0) {
            bulk_load(place, rec, LQ_KV_HEAD + LQ_KV_BLOCK * DP, bar);
          } else {
            bulk_load(place, rec, LQ_KV_HEAD, bar);
            bulk_load(place + LQ_KV_HEAD, rec + LQ_KV_HEAD + LQ_KV_BLOCK * DP, LQ_KV_BLOCK * DP, bar);
          }
        }
      };
      ask(ow);
      const uint8_t* now = find(ow);
      fetch(ow, now);
      ask(ow + OPEN_WARPS);
      int asked = now ? 1 : 0, had = 0;                      // copies that were asked for, that have come
      for (int n = ow; n < 8 * tiles; n += OPEN_WARPS) {
        const int j = n >> 3, st = j & 1, side = n >> 2 & 1, w = n & 3;
        const uint8_t* next = find(n + OPEN_WARPS);
        ask(n + 2 * OPEN_WARPS);
        uint32_t head = 0;
        if (now) {
          if (!wait(c.raw[ow], had, LQ_STAGE_PRODUCER)) break;
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(head) : "r"(place) : "memory");
          ++had;
        }
        if (j >= 2 && !wait(side == 0 ? c.k_empty[st] : c.v_empty[st], (j >> 1) - 1, LQ_STAGE_PRODUCER)) break;
        if (side == 0 && lane == 0) c.missing[j & 3][w] = !now;
        const auto then = [&]() {                            // what the warp's place held is in registers
          fetch(n + OPEN_WARPS, next);
          asked += next ? 1 : 0;
        };
        if (!now) {
          then();
          zero_rows(smem_u32(side == 0 ? sk : sv) + st * (side == 0 ? k_bytes(DP) : v_bytes(DP)), w, side, DP, lane);
        } else if (side == 0) {
          open_keys<NK>(place + LQ_KV_HEAD, smem_u32(sk) + st * k_bytes(DP) + 32 * w * 128, head, lane, then);
        } else {
          open_values<NK>(place + LQ_KV_HEAD, smem_u32(sv) + st * v_bytes(DP) + w / 2 * DP * 128, head >> 8, w & 1, lane, then);
        }
        fence_proxy_async();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(side == 0 ? &c.k_full[st] : &c.v_full[st]));
        now = next;
      }
      // (a wait gave up: what is in flight lands before the block leaves)
      if (!good && asked > had) mbar_settle(bar, (asked - 1) & 1);
    } else if (tiles > 0) {
      const uint32_t idesc_s = IDESC_F16 | idesc_shape(KV), idesc_o = IDESC_F16 | idesc_shape(DP);
      const auto product_s = [&](int half, int st) {         // by one thread
        const uint32_t a = smem_u32(sq + half * q_bytes(DP)), b = smem_u32(sk + st * k_bytes(DP));
#pragma unroll
        for (int x = 0; x < NK; ++x)
          tc_mma<TC_F16>(tmem + COL_S + half * 128, make_smem_desc(a + x / 4 * TILE * 128 + x % 4 * 32), make_smem_desc(b + x / 4 * KV * 128 + x % 4 * 32), idesc_s,
                         x > 0);
      };
      const auto product_o = [&](int half, int st, int piece, bool add) {          // of a piece
        const uint32_t b = smem_u32(sv + st * v_bytes(DP));
#pragma unroll
        for (int y = 0; y < PIECE / 16; ++y) {
          const int x = PIECE / 16 * piece + y;
          tc_mma_ta(tmem + COL_O + half * 128, tmem + COL_S + half * 128 + 8 * x, make_smem_desc(b + x / 4 * DP * 128 + x % 4 * 32), idesc_o, add || y > 0);
        }
      };
      wait(c.k_full[0], 0, LQ_STAGE_MMA);
      for (int half = 0; half < halves; ++half) {
        if (!wait(c.q_full[half], 0, LQ_STAGE_MMA)) break;
        tc_fence_after();
        if (elect_one()) {
          product_s(half, 0);
          tc_commit(smem_u32(&c.s_full[half]));
          if (half == halves - 1) tc_commit(smem_u32(&c.k_empty[0]));
        }
        __syncwarp();
      }
      for (int j = 0; j < k.tiles && good; ++j) {
        const int st = j & 1, next = st ^ 1;
        const bool last = j == k.tiles - 1;
        for (int half = 0; half < halves; ++half) {
          if (half == 0 && !wait(c.v_full[st], j >> 1, LQ_STAGE_MMA)) break;
          if (half == 0 && !last && !wait(c.k_full[next], (j + 1) >> 1, LQ_STAGE_MMA)) break;
#pragma unroll
          for (int x = 0; x < PIECES - 1; ++x) {
            if (!wait(c.p_full[half][x], j, LQ_STAGE_MMA)) break;
            tc_fence_after();
            if (elect_one()) product_o(half, st, x, j > 0 || x > 0);
            __syncwarp();
          }
          if (!wait(c.p_full[half][PIECES - 1], j, LQ_STAGE_MMA)) break;
          tc_fence_after();
          if (elect_one()) {
            product_o(half, st, PIECES - 1, true);
            if (half == halves - 1) tc_commit(smem_u32(&c.v_empty[st]));
            if (last) {
              tc_commit(smem_u32(&c.o_full[half]));
            } else {
              product_s(half, next);
              tc_commit(smem_u32(&c.s_full[half]));
              if (half == halves - 1) tc_commit(smem_u32(&c.k_empty[next]));
            }
          }
          __syncwarp();
        }
      }
      if (!good) {                                           // a wait gave up: what has been issued gets a bounded time to end
        if (elect_one()) tc_commit(smem_u32(&c.q_full[0]));
        __syncwarp();
        mbar_settle(smem_u32(&c.o_full[0]), 0);
      }
    }
  }
  __syncthreads();
  if (warp == MMA_WARP) {
    tc_fence_after();
    tmem_dealloc(tmem, TMEM_COLS);
  }
}

// Joins the parts of tiles that were shared out: 32 rows a thread block, a row a lane, entries by warps, every load a line of 128 bytes.
constexpr int JOIN_WARPS = 8, JOIN_ROWS = 32;
template <int NK>
__global__ void __launch_bounds__(32 * JOIN_WARPS) lq_attn_join_kernel(const __grid_constant__ LqAttnParams p) {
  constexpr int DP = 16 * NK, STEP = 2 * TILE;
  const int warp = threadIdx.x >> 5, row = blockIdx.y * JOIN_ROWS + (threadIdx.x & 31);
  grid_launch_dependents();
  grid_dependency_wait();
  const int4 meta = p.tile_meta[blockIdx.x];
  const int parts = meta.x;
  if (parts < 2 || row >= meta.w) return;
  const float* from = p.tile_part + (long long)blockIdx.x * p.splits * (DP + 2) * STEP + row;
  constexpr long long PART = (DP + 2) * STEP;
  const float scale = lq_attn_scale(p);
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i < parts; ++i) m = fmaxf(m, from[i * PART + DP * STEP]);
  const float ref = m > -INFINITY ? m : 0.f;
  float2 o[NK];
#pragma unroll
  for (int g = 0; g < NK; ++g) o[g] = make_float2(0.f, 0.f);
  for (int i = 0; i < parts; ++i) {
    const float* at = from + i * PART;
    const float by = ex2((at[DP * STEP] - ref) * scale);
    l = fmaf(by, at[(DP + 1) * STEP], l);
#pragma unroll
    for (int g = 0; g < NK; ++g) {                         // entries 16 g + 2 warp and the next
      o[g].x = fmaf(by, at[(16 * g + 2 * warp) * STEP], o[g].x);
      o[g].y = fmaf(by, at[(16 * g + 2 * warp + 1) * STEP], o[g].y);
    }
  }
  const float by = l > 0.f ? 16.f / l : 0.f;
  const int place = (p.whole + blockIdx.x) % p.b.heads, r = meta.z + row, tok = r / p.group;
  __half* out = p.out + (meta.y + tok) * p.out_row + (long long)(place * p.group + r - tok * p.group) * p.out_head;
#pragma unroll
  for (int g = 0; g < NK; ++g)
    if (16 * g + 2 * warp < p.D) *reinterpret_cast<uint32_t*>(out + 16 * g + 2 * warp) = pack(o[g].x * by, o[g].y * by);
}

constexpr size_t tile_smem(int Dp) { return 2 * (size_t)(q_bytes(Dp) + k_bytes(Dp) + v_bytes(Dp)) + OPEN_WARPS * raw_bytes(Dp) + sizeof(Control); }

static_assert(tile_smem(128) <= 232448, "");

template <typename F>
auto with_size(int Dp, const F& f) {
  switch (Dp) {
    case 64: return f(lq_attn_tile_kernel<4>, lq_attn_join_kernel<4>);
    case 80: return f(lq_attn_tile_kernel<5>, lq_attn_join_kernel<5>);
    case 96: return f(lq_attn_tile_kernel<6>, lq_attn_join_kernel<6>);
    case 112: return f(lq_attn_tile_kernel<7>, lq_attn_join_kernel<7>);
    default: return f(lq_attn_tile_kernel<8>, lq_attn_join_kernel<8>);
  }
}

}  // namespace

lq_status lq_attn_tile_prepare(const lq_kvcache* C) {
  return with_size(C->Dp, [&](auto* kernel, auto*) {
    cudaFuncAttributes at;
    if (lq_note_cuda(cudaFuncGetAttributes(&at, kernel)) != cudaSuccess) return LQ_ERR_CUDA;
    if (at.numRegs < LAUNCH_REGS) return LQ_ERR_UNSUPPORTED;
    return lq_note_cuda(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)tile_smem(C->Dp))) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
  });
}

lq_status lq_attn_tile_launch(const lq_kvcache* C, LqAttnParams p, cudaStream_t st) {
  // tiles of 256 rows: exactly so many where all sequences have as many rows; else at most one of each sequence is not full
  const long long units = (p.b.row_start ? (long long)p.b.rows * p.group / (2 * TILE) + p.b.sequences
                                         : p.b.sequences * (((long long)p.b.each * p.group + 2 * TILE - 1) / (2 * TILE))) * C->heads;
  if (units > 0x7fffffffll) return LQ_ERR_UNSUPPORTED;
  // Where the last of them leave SMs idle, as many thread blocks to each of these as there is room for, unless no sequence is long (us of 512 tiles, one
  // block each / the last 68 shared by two: 4096 tokens, heads of 72 273 / 254; 4096 behind 4096, causal, heads of 128 448 / 422).
  p.whole = (int)(units / C->sms * C->sms);
  const int last = (int)(units - p.whole);
  p.splits = last > 0 && (long long)p.b.page_stride * C->page_tokens >= 4 * MIN_TILES * KV ? C->sms / last : 1;
  if (p.splits == 1) p.whole = (int)units;
  const cudaError_t e = with_size(C->Dp, [&](auto* kernel, auto* join) {
    const int split = (int)units - p.whole;
    const cudaError_t first = lq_launch(kernel, p.whole + split * p.splits, THREADS, tile_smem(C->Dp), st, p);
    if (first != cudaSuccess || split == 0) return first;
    return lq_launch_grid(join, dim3((unsigned)split, 2 * TILE / JOIN_ROWS), 32 * JOIN_WARPS, 1, 0, st, p);
  });
  return lq_note_cuda(e) == cudaSuccess ? LQ_OK : LQ_ERR_CUDA;
}
