// How a launch of the heads kernel shares out its rows and heads.  Host arithmetic only, apart from the launch so that a test can compile it
// by itself.  Internal: not part of the C ABI.
#pragma once

#include <algorithm>

constexpr int LQ_HEADS_WARPS = 4, LQ_HEADS_ROWS = 2;         // warps of a block; most rows of one

struct LqHeadsCut {
  int walk, parts[2];          // heads a warp walks over at a time, and the parts that makes of Q's and K's
  int block_rows, blocks, blocks_y;
};

// A warp walks over all heads of a side, or over as many as the shorter side has (at least four steps of `groups` heads), so that warps have
// like work, once there are rows enough to fill the GPU (24 warps an SM); below that over fewer, down to one step.
inline LqHeadsCut lq_heads_cut(int rows, int heads0, int heads1, int groups, int sms) {
  LqHeadsCut c;
  const int fill = sms * 24;
  int walk = std::max(heads0, heads1);
  if (heads0 > 0 && heads1 > 0) walk = std::min(walk, std::max(4 * groups, std::min(heads0, heads1)));
  const auto parts = [&](int w) { return (heads0 + w - 1) / w + (heads1 + w - 1) / w; };
  int low = 1, high = (walk + groups - 1) / groups;          // the longest walk, in steps, that fills, or one
  while (low < high) {
    const int mid = (low + high + 1) / 2;
    if ((long long)rows * parts(mid * groups) < fill) high = mid - 1;
    else low = mid;
  }
  c.walk = low * groups;
  c.parts[0] = (heads0 + c.walk - 1) / c.walk;
  c.parts[1] = (heads1 + c.walk - 1) / c.walk;
  const int n = c.parts[0] + c.parts[1], few = fill / LQ_HEADS_WARPS;
  c.block_rows = std::max(1, std::min(LQ_HEADS_ROWS, rows / few));
  c.blocks = 1 + (rows - 1) / c.block_rows;                  // (up to 2^31 - 1 rows: no sum beyond them)
  c.blocks_y = std::max(1, std::min((c.block_rows * n + LQ_HEADS_WARPS - 1) / LQ_HEADS_WARPS, few / c.blocks));
  return c;
}
