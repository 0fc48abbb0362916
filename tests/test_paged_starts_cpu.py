"""The split of a paged decode call whose caches' starts count as rounds, walked on the CPU as its kernels walk it
(the header that they share is compiled with the host compiler)."""
import ctypes
import random
import shutil
import subprocess

import pytest

from paper_2406_14909_amd import build as B

pytestmark = pytest.mark.skipif(shutil.which(B.CXX) is None, reason="no host compiler")

_CODE = r"""
#include <vector>
#include "paged_split.h"
using namespace moa;

// Caches of rounds[0 .. pairs - 1]: 0 when every round of the keys is read once, in its order, a cache
// is written as a whole by the one worker that has all of it, and the others' pieces are those that the merge looks for;
// else the broken rule.
extern "C" int walk(int pairs, const uint32_t* rounds, uint32_t slots, uint32_t* out) {
  uint32_t units = 0, longest = 0;
  for (int i = 0; i < pairs; ++i) {
    units += rounds[i];
    longest = std::max(longest, rounds[i]);
  }
  const uint32_t start = paged_start_rounds(units, pairs, slots);
  out[0] = start;
  if (start > 1 || (start == 1) != (uint32_t(pairs) >= slots && units >= 2u * pairs)) return 1;
  if (start == 0) return 0;
  const PagedSplit s = paged_split(units + pairs * start, longest + start, slots);
  if (s.workers < 1 || s.workers > slots) return 2;
  std::vector<uint32_t> read(pairs, 0), first(pairs, ~0u), last(pairs, 0), parts(pairs, 0);
  std::vector<char> wrote(pairs, 0);
  int pair = 0;
  uint32_t at = 0;                                       // rounds in front of the pair
  out[1] = 0;
  for (uint32_t w = 0; w < s.workers; ++w) {
    uint32_t x = s.start(w);
    const uint32_t end = s.start(w + 1);
    while (x < end) {
      const uint32_t n = rounds[pair] + start, lo = x - at, hi = std::min(n, lo + (end - x));
      const PagedPart part(lo, hi, n, start);
      if (part.first > part.last || part.last > rounds[pair]) return 3;
      if (part.last > part.first) {
        if (part.first != read[pair]) return 4;
        read[pair] = part.last;
        first[pair] = std::min(first[pair], w);
        last[pair] = w;
        ++parts[pair];
        if (part.whole) wrote[pair] = 1;
        if (part.whole != (part.first == 0 && part.last == rounds[pair])) return 5;
      } else if (part.last > 0) {
        return 6;                                        // a piece of no keys that would be taken for one
      }
      if (lo < start && hi <= start && hi < n) ++out[1];  // a start alone, its keys with the next worker
      x += hi - lo;
      if (hi == n) {
        at += n;
        ++pair;
      }
    }
  }
  if (pair != pairs) return 7;
  at = 0;
  for (int i = 0; i < pairs; ++i) {
    if (read[i] != rounds[i]) return 8;
    if (rounds[i] > 0) {
      const uint32_t x0 = at + start, w0 = s.worker_of(x0), w1 = s.worker_of(x0 + rounds[i] - 1);    // the merge's
      if (w0 != first[i] || w1 != last[i] || parts[i] != w1 - w0 + 1) return 9;
      if ((w0 == w1) != (wrote[i] == 1)) return 10;
    }
    at += rounds[i] + start;
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("starts")
    src, so = d / "walk.cpp", d / "walk.so"
    src.write_text(_CODE)
    subprocess.run([B.CXX, "-std=c++17", "-O1", "-shared", "-fPIC", f"-I{B.INCLUDE}", f"-I{B.CSRC}", str(src), "-o",
                    str(so)], check=True)
    return ctypes.CDLL(str(so))


def test_caches_whose_starts_count(lib):
    rng = random.Random(4)
    counted = alone = 0
    for _ in range(1500):
        pairs = rng.choice([1, 2, 8, 33, 256, 511, 512, 513, 1500])
        top = rng.choice([1, 3, 8, 40, 1200])
        rounds = [rng.choice([0, 1, rng.randint(0, top), rng.randint(top // 2, top)]) for _ in range(pairs)]
        slots = rng.choice([1, 2, 7, 64, 256, 512])
        out = (ctypes.c_uint32 * 2)()
        assert lib.walk(pairs, (ctypes.c_uint32 * pairs)(*rounds), slots, out) == 0, (pairs, top, slots, rounds[:9])
        counted += out[0]
        alone += out[1] if out[0] else 0
    assert counted > 300 and alone > 300


def test_when_they_count(lib):
    out = (ctypes.c_uint32 * 2)()
    for pairs, each, slots, want in ((512, 2, 512, 1), (511, 2, 512, 0), (512, 1, 512, 0), (600, 1000, 512, 1), (1, 2, 1, 1)):
        assert lib.walk(pairs, (ctypes.c_uint32 * pairs)(*[each] * pairs), slots, out) == 0 and out[0] == want, (pairs, each)
