"""The work split of a paged decode call, walked on the CPU as its kernels walk it: the
header that they share is compiled with the host compiler.  Every visible key of every
cache is read exactly once, at its own position; a cache cut over several workers finds
its partial results in slots of its own; pieces differ by at most one round; a token that
sees nothing has a worker that writes its zeros."""
import ctypes
import os
import random
import shutil
import subprocess

import pytest

import oracle
from paper_2406_14909_amd import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.CXX) is None, reason="no host compiler")

_CODE = r"""
#include <vector>
#include "paged_split.h"
using namespace moa;

// Positions of the visible keys of one query, and the table index of each one's page as
// the kernels find it (by page number); returns their number.
extern "C" int keys(int pos, int window, int shift, int sink, int from, int capacity, int page_shift, int* at, int* page) {
  const VisibleKeys v = visible_keys(pos, window, shift, sink, from, capacity);
  const VisiblePages p(v, page_shift);
  int last = -1;
  for (int x = 0; x < v.count; ++x) {
    at[x] = v.at(x);
    const int n = p.number(x < v.sinks, v.at(x) >> page_shift);
    if (n < last || n > last + 1) return -1;                 // page numbers rise by at most one
    last = n;
    page[x] = p.index(n);
  }
  return v.count;
}

// 0 when the split of caches of rounds[0 .. pairs - 1] is sound, else the broken rule.
extern "C" int walk(int pairs, const uint32_t* rounds, uint32_t slots, uint32_t* out) {
  uint32_t units = 0, longest = 0;
  for (int i = 0; i < pairs; ++i) {
    units += rounds[i];
    longest = std::max(longest, rounds[i]);
  }
  const PagedSplit s = paged_split(units, longest, slots);
  if (units == 0) return s.workers == 0 ? 0 : 1;
  if (s.workers < 1 || s.workers > slots || s.start(0) != 0 || s.start(s.workers) != units) return 2;
  std::vector<char> used(size_t(s.workers) + pairs, 0);
  uint32_t most = 0, least = ~0u;
  for (uint32_t w = 0; w < s.workers; ++w) {
    const uint32_t n = s.start(w + 1) - s.start(w);
    if (n == 0 || s.start(w + 1) < s.start(w)) return 3;
    most = std::max(most, n);
    least = std::min(least, n);
  }
  if (most > least + 1) return 4;
  uint32_t x = 0, parts = 0;
  for (int i = 0; i < pairs; ++i) {
    if (rounds[i] == 0) continue;
    const uint32_t w0 = s.worker_of(x), w1 = s.worker_of(x + rounds[i] - 1);
    for (uint32_t r = 0; r < rounds[i]; ++r) {
      const uint32_t w = s.worker_of(x + r);
      if (s.start(w) > x + r || s.start(w + 1) <= x + r) return 5;
    }
    for (uint32_t w = w0; w <= w1 && w0 != w1; ++w)
      if (used[size_t(w) + i]++) return 6;
    parts = std::max(parts, w1 - w0 + 1);
    x += rounds[i];
  }
  out[0] = s.workers;
  out[1] = parts;
  return 0;
}

// Row tiles of pairs (tokens, position, window) cut for `slots` workers: 0 when every key tile
// of every row tile is walked once, the merge finds all pieces in slots of their own, and no
// piece costs more than its share.  tiles[i]: key tiles of a row tile, by some rule.
extern "C" int row_walk(int pairs, const int64_t* tokens, const int* pos, const int* window, int sink, int gs, int rows,
                        int64_t cap, int least, int log_slots, int* out) {
  std::vector<PairCost> cost;
  std::vector<int64_t> at;
  int64_t units = 0;
  for (int i = 0; i < pairs; ++i) {
    cost.push_back(pair_cost(tokens[i], pos[i], window[i], 0, sink, gs, rows, cap));
    const PairCost& c = cost.back();
    if (c.before(0) != 0) return 1;
    const int step = rows >> gs;
    int64_t sum = 0;
    for (int k = 0; k < c.tiles && k < 300; ++k) {
      int64_t end = int64_t(c.first) + step * (k + 1);
      sum += kTileCost + std::min<int64_t>(end, c.most);
      if (c.before(k + 1) != sum) return 2;
    }
    if (c.tiles > 0 && int64_t(c.tiles) * step < tokens[i]) return 3;
    at.push_back(units);
    units += c.before(c.tiles);
  }
  const RowSplit s = row_split(units, least, log_slots);
  const int workers = s.workers();
  if (units == 0) return workers == 0 ? 0 : 4;
  if (workers < 1 || workers > 1 << log_slots || s.start(0) != 0 || s.start(workers) != units) return 5;
  if (workers > 1 && units / workers < least) return 10;
  std::vector<char> used(2 * size_t(workers), 0);
  int parts = 0;
  for (int i = 0; i < pairs; ++i) {
    for (int k = 0; k < cost[i].tiles; ++k) {
      const int64_t c0 = at[i] + cost[i].before(k), c1 = at[i] + cost[i].before(k + 1);
      const int w0 = s.worker_of(c0), w1 = s.worker_of(c1 - 1);
      const int n = 1 + (k * 7 + i) % 50;                     // key tiles
      int next = 0;
      for (int w = w0; w <= w1; ++w) {
        const int64_t x = std::max(c0, s.start(w)), end = std::min(c1, s.start(w + 1));
        if (end <= x) return 6;
        const int t0 = row_part(n, x - c0, c1 - c0), t1 = row_part(n, end - c0, c1 - c0);
        if (t0 != next || t1 < t0) return 7;
        next = t1;
        if (w0 != w1) {
          const size_t slot = 2 * size_t(w) + (x == c0 ? 1 : 0);
          if ((w == w0) != (x == c0) || used[slot]++) return 8;
        }
      }
      if (next != n) return 9;
      parts = std::max(parts, w1 - w0 + 1);
    }
  }
  out[0] = workers;
  out[1] = parts;
  return 0;
}

extern "C" uint32_t rounds(int pos, int count, int shift, int merge) { return paged_rounds(pos, count, shift, merge != 0); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    src, so = d / "walk.cpp", d / "walk.so"
    src.write_text(_CODE)
    subprocess.run([B.CXX, "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{B.INCLUDE}", f"-I{B.CSRC}", str(src), "-o",
                    str(so)], check=True)
    return ctypes.CDLL(str(so))


def test_visible_keys_are_the_oracles(lib):
    rng = random.Random(1)
    for _ in range(3000):
        ps = rng.choice([4, 5, 6, 8])
        capacity = rng.randint(1, 30) << ps
        pos = rng.randint(0, min(capacity + 50, 1500))
        w, s = rng.choice([1, 2, 17, 64, 100, 500, 5000]), rng.choice([0, 1, 4, 64, 70, 3000])
        block = rng.choice([0, 64])
        start = rng.choice([0, 0, 1, 63, 64, 100, pos, pos + 1, capacity])
        at, page = (ctypes.c_int * 4000)(), (ctypes.c_int * 4000)()
        n = lib.keys(pos, -(-w // 64) if block else w, 6 if block else 0, s, start, capacity, ps, at, page)
        ref = [j for j in oracle.visible_set(pos, w, s, block).tolist() if start <= j < capacity]
        assert list(at[:max(n, 0)]) == ref, (pos, w, s, block, start, capacity)
        assert list(page[:n]) == [j >> ps for j in ref]


def test_every_round_is_read_once_and_partials_have_slots(lib):
    rng = random.Random(2)
    for i in range(600):
        pairs = rng.choice([1, 2, 8, 33, 256, 1500])
        top = rng.choice([1, 3, 40, 1200])
        rounds = [rng.choice([0, 1, rng.randint(0, top)]) for _ in range(pairs)]
        out = (ctypes.c_uint32 * 2)()
        slots = rng.choice([1, 2, 64, 512, 768, 2048])
        assert lib.walk(pairs, (ctypes.c_uint32 * pairs)(*rounds), slots, out) == 0, (pairs, top, slots)
        assert not any(rounds) or out[1] <= 2 * 256


def test_rounds(lib):
    assert [lib.rounds(-1, 0, 7, m) for m in (0, 1)] == [0, 0]
    assert [lib.rounds(5, 0, 7, m) for m in (0, 1)] == [1, 0]
    assert [lib.rounds(5, n, 7, 0) for n in (1, 128, 129)] == [1, 1, 2]


def test_every_key_tile_of_a_row_tile_is_walked_once(lib):
    rng = random.Random(3)
    for _ in range(500):
        pairs = rng.choice([1, 3, 8, 64])
        tokens = [rng.choice([0, 1, 5, 128, rng.randint(1, 20000)]) for _ in range(pairs)]
        pos = [rng.choice([-1, 0, 0, 100, rng.randint(0, 200000), 2 ** 31 - 5]) for _ in range(pairs)]
        window = [rng.choice([1, 64, 1000, rng.randint(1, 100000)]) for _ in range(pairs)]
        rows = rng.choice([32, 128])
        cap = rng.choice([64, 5000, 1 << 20, 1 << 30])
        out = (ctypes.c_int * 2)()
        args = ((ctypes.c_int64 * pairs)(*tokens), (ctypes.c_int * pairs)(*pos), (ctypes.c_int * pairs)(*window))
        assert lib.row_walk(pairs, *args, rng.choice([0, 64, 3000]), rng.choice([0, 1, 2, 3]), rows, ctypes.c_int64(cap),
                            rng.choice([1, 128, 512]), rng.choice([0, 6, 9]), out) == 0, (tokens, pos, window, rows, cap)
