"""How attention's records are shared out over a grid, on the CPU: every record once, what is one block's as a whole, and who joins what is not."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include <algorithm>
#include "lq_attn_places.h"
struct None {};
using Place = LqAttnPlace<None>;
// The kernel's steps for one block: its records' numbers (sequence, head, tile, record) warp after warp into `out`, its edges; returns how many.
extern "C" int block(const int* tiles, const int* each, int sequences, int heads, int warps, int grid, int small, int threads, int b, long long* edges,
                     long long* share_out, int* out) {
  const auto measure = [&](int s) { Place p = {}; p.s = s; p.tiles = tiles[s]; p.each = tiles[s] ? each[s] : 0; return p; };
  long long total = 0;
  for (int s = 0; s < sequences; ++s) total += lq_attn_records(measure(s), heads);
  long long all_tiles = 0;
  for (int s = 0; s < sequences; ++s) all_tiles += (long long)tiles[s] * heads;
  const LqAttnCut cut = lq_attn_cut(total, all_tiles, grid, warps);
  *share_out = cut.parted ? 0 : cut.share;
  const long long share = cut.share;
  Place found = {};
  edges[0] = edges[1] = cut.parted ? 0 : total;
  edges[2] = 0; edges[3] = 1;
  const int chunk = (sequences + threads - 1) / threads;
  long long begin = 0;
  for (int first = 0; first < sequences; first += chunk) {           // a thread
    long long sum = 0;
    for (int s = first; s < std::min(sequences, first + chunk); ++s) sum += lq_attn_count(measure(s), heads, cut, small);
    if (cut.parted && b >= begin && b < begin + sum) {
      Place at = measure(first);
      int part, parts;
      edges[1] = lq_attn_part(at, begin, b, heads, small, cut, part, parts, measure);
      edges[2] = part; edges[3] = parts;
      found = at;
    }
    if (!cut.parted)
    for (int i = 0; i < 2; ++i) {
      const long long edge = (b + i) * share;
      if (edge < begin || edge >= begin + sum) continue;
      Place at = measure(first);
      edges[i] = lq_attn_edge(at, begin, edge, heads, small, measure);
      if (i == 0) {
        if (edges[0] < total) lq_attn_walk(at, 0, heads, sequences, measure);
        found = at;
      }
    }
    begin += sum;
  }
  int n = 0;
  for (int w = 0; w < warps; ++w) {
    long long left = (edges[1] - edges[0] - w + warps - 1) / warps;
    Place at = found;
    if (left > 0 && !lq_attn_walk(at, w, heads, sequences, measure)) return -1;
    for (; left > 0; --left) {
      out[4 * n] = at.s; out[4 * n + 1] = at.head; out[4 * n + 2] = at.tile; out[4 * n++ + 3] = at.i;
      if (left > 1 && !lq_attn_walk(at, warps, heads, sequences, measure)) return -1;
    }
  }
  return n;
}
extern "C" long long quotient(long long a, long long b) { return lq_quotient(a, b); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("places")
    (d / "p.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", os.path.join(ROOT, "paper_2604_18117_b200", "csrc"),
                    str(d / "p.cpp"), "-o", str(d / "p.so")], check=True)
    so = C.CDLL(str(d / "p.so"))
    so.quotient.restype, so.quotient.argtypes = C.c_longlong, [C.c_longlong] * 2
    return so


def shared_out(so, tiles, each, heads, warps, grid, small, threads):
    tiles, each = np.array(tiles, np.int32), np.array(each, np.int32)
    total = int((tiles.astype(np.int64) * each * heads).sum())
    seen, owners, parts_of, edges, share = {}, {}, {}, (C.c_longlong * 4)(), C.c_longlong()
    out, ends = np.zeros((total + 1, 4), np.int32), 0
    for b in range(grid):
        n = so.block(tiles.ctypes.data_as(C.c_void_p), each.ctypes.data_as(C.c_void_p), len(tiles), heads, warps, grid, small, threads, b, edges, C.byref(share),
                     out.ctypes.data_as(C.c_void_p))
        assert n == max(0, edges[1] - edges[0]), (b, n, list(edges))
        parted = share.value == 0
        if parted:
            parts_of.update({tuple(r[:3]): (b - edges[2], edges[3]) for r in out[:n].tolist()})
            assert n == 0 or len({tuple(r[:3]) for r in out[:n].tolist()}) == 1          # of one tile
        else:
            assert edges[0] >= ends
            ends = max(ends, edges[1])
        for s, h, t, i in out[:n].tolist():
            assert (s, h, t, i) not in seen
            seen[s, h, t, i] = b
            owners.setdefault((s, h, t), set()).add(b)
    assert len(seen) == total and (parted or ends == total)
    at = 0
    for s in range(len(tiles)):
        for h in range(heads):
            for t in range(tiles[s]):
                assert [(s, h, t, i) in seen for i in range(each[s])] == [True] * each[s]
                who = owners[s, h, t]
                if each[s] <= small:
                    assert len(who) == 1
                elif parted:
                    first, parts = parts_of[s, h, t]
                    assert who == set(range(first, first + parts))
                elif len(who) > 1:                         # those that the joining block counts on
                    assert who == set(range(at // share.value, (at + each[s] - 1) // share.value + 1))
                at += int(each[s])


def test_batches_of_all_kinds(lib):
    rng = np.random.default_rng(2)
    for _ in range(400):
        S = int(rng.integers(1, 40))
        tiles = rng.integers(0, 4, S) if rng.random() < 0.7 else np.ones(S, int)
        each = rng.integers(1, int(rng.choice([3, 20, 40, 200])), S)
        if not tiles.any():
            tiles[int(rng.integers(S))] = 1
        warps = int(rng.choice([4, 8]))
        shared_out(lib, tiles, each, int(rng.integers(1, 9)), warps, int(rng.choice([1, 7, 148])), int(rng.choice([0, 2, 4])) * warps, int(rng.choice([4, 32, 256])))


@pytest.mark.parametrize("tiles,each,heads", [([1], [1], 1), ([1], [10], 16), ([1], [4096], 8), ([0, 0, 1], [5, 5, 5], 1), ([1, 0, 0, 1], [33, 1, 1, 33], 3),
                                              ([9], [4], 2), ([1] * 64, [256 - 3 * i for i in range(64)], 8), ([2] * 24, [34] * 24, 2)])
def test_batches_that_programs_have(lib, tiles, each, heads):
    for warps, threads in ((8, 256), (4, 128)):
        shared_out(lib, tiles, each, heads, warps, 148, 4 * warps, threads)


def test_quotients_of_large_numbers(lib):
    for a in (0, 1, 2 ** 32 - 1, 2 ** 32, 2 ** 40 + 12345):
        for b in (1, 7, 2 ** 32 - 1, 2 ** 33):
            assert lib.quotient(a, b) == a // b
