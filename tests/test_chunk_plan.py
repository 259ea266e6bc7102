"""How a batch of chunk_attention becomes pieces (chunk_plan.h, no device types), compiled and
counted on the CPU as the kernel's waves count them: whatever offsets and lengths the device holds,
the parts' places and the split items' records fit the workspace, and where records are
published every piece has a workgroup, so that each record has its writer."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_29364_amd", "csrc")

SOURCE = r"""
#include <cmath>
#include <vector>
#include "chunk_plan.h"

// The counts of find_piece() for host copies of a batch's arrays.  trusting: as if the offsets rose
// whatever they hold.  out: grid, places the workspace has, records it has; items, pieces, places,
// split items of the device.
extern "C" void count(const int32_t* indptr, const int32_t* lens, int bs,
                      int total_q, int hq, int hkv, int max_len, int trusting, int64_t* out) {
  const Plan p = plan(bs, total_q, hq, hkv, max_len);
  auto clamp = [](int64_t x, int64_t hi) { return std::min(std::max(x, (int64_t)0), hi); };
  int64_t items = 0, places = 0, split_items = 0, n = 0;
  float total = 0.f;
  bool rising = true;
  std::vector<int> tiles(bs), stages(bs), splits(bs, 1);
  for (int r = 0; r < bs; ++r) {
    const int64_t a = clamp(indptr[r], total_q), raw = clamp(indptr[r + 1], total_q);
    rising &= raw >= a;
    const int64_t b = std::max(raw, a), length = clamp(lens[r], max_len);
    tiles[r] = (int)(((b - a) * (hq / hkv) + p.tile - 1) / p.tile);
    stages[r] = (int)std::max<int64_t>((length + kStage - 1) / kStage, 1);
    items += tiles[r];
    total += (float)tiles[r] * stages[r];
  }
  rising |= trusting != 0;
  Tail tail{0, 1};
  if (p.places) {
    const float limit = rising ? split_limit((int)items, total, hkv) : INFINITY;
    for (int r = 0; r < bs; ++r) {
      splits[r] = parts_of(stages[r], limit);
      if (splits[r] > 1) places += tiles[r] * splits[r], split_items += tiles[r];
    }
    if (places > p.places) {
      std::fill(splits.begin(), splits.end(), 1);
      split_items = 0;
    }
    if (rising && split_items == 0) {
      tail = last_round((int)items, hkv);
      split_items = tail.items;
      places = (int64_t)tail.items * tail.parts;
    }
  }
  for (int r = 0; r < bs; ++r) n += (int64_t)tiles[r] * splits[r];
  n += (int64_t)tail.items * (tail.parts - 1);
  const int64_t o[] = {pieces(p, hkv), p.places, p.split_items, items, n, places, split_items};
  std::copy(o, o + 7, out);
}
"""


@pytest.fixture(scope="module")
def count(tmp_path_factory):
    cxx = shutil.which(os.environ.get("CXX", "g++")) or shutil.which("c++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    d = tmp_path_factory.mktemp("chunk_plan")
    (d / "count.cpp").write_text(SOURCE)
    subprocess.run([cxx, "-std=c++17", "-shared", "-fPIC", f"-I{CSRC}", str(d / "count.cpp"), "-o",
                    str(d / "count.so")], check=True)
    f = ctypes.CDLL(str(d / "count.so")).count

    def call(indptr, lens, total_q, hq, hkv, max_len, trusting=0):
        a, b = (np.ascontiguousarray(x, np.int32) for x in (indptr, lens))
        out = (ctypes.c_int64 * 7)()
        f(a.ctypes.data_as(ctypes.c_void_p), b.ctypes.data_as(ctypes.c_void_p), len(b),
          int(total_q), hq, hkv, int(max_len), trusting, out)
        return dict(zip(("grid", "room", "records", "items", "pieces", "places", "split"), out))
    return call


def sound(c):
    return c["split"] == 0 or (c["pieces"] <= c["grid"] and c["places"] <= c["room"]
                               and c["split"] <= c["records"])


# batches of two requests that count the same rows over and over
FALLING = [([0, 1120, 0, 1120], [1024] * 3, 1120, 32, 8, 1024),
           ([0, 300] * 128 + [0], [4000] * 256, 300, 4, 2, 5000),
           ([0, 2000, 5, 2000, 7, 2000], [9000] * 5, 2000, 32, 8, 9000)]


@pytest.mark.parametrize("case", FALLING)
def test_falling_offsets_are_not_split(count, case):
    c = count(*case)
    assert c["items"] > c["grid"] - c["room"] and sound(c) and c["split"] == 0
    # taken as if they rose, two of the batches publish records without a writer
    assert case is FALLING[2] or not sound(count(*case, trusting=1))


def test_any_contents(count):
    rng = np.random.default_rng(0)
    unsound = split = last = 0
    for _ in range(6000):
        bs = int(rng.choice([1, 2, 3, 5, 17, 63, 64, 65, 200, 256]))
        hkv = int(rng.choice([1, 2, 3, 4, 8, 12, 32, 100, 256]))
        hq = hkv * int(rng.choice([1, 2, 3, 4, 7, 16]))
        max_len = int(2 ** rng.uniform(0, 17))
        total = int(2 ** rng.uniform(0, 14))
        rising = rng.random() < 0.5
        indptr = rng.integers(-5 if not rising else 0, total + 1, bs + 1)
        if rng.random() < 0.5:
            indptr = np.where(rng.random(bs + 1) < 0.5, 0, total)
        if rising:
            indptr = np.sort(indptr)
        lens = np.minimum(2 ** rng.uniform(0, 18, bs), 2**31 - 1).astype(np.int64)
        if rng.random() < 0.5:
            lens[:] = max_len
        c = count(indptr, lens, total, hq, hkv, max_len)
        assert sound(c), (bs, hkv, hq, max_len, total, indptr.tolist(), lens.tolist(), c)
        if rising:
            assert c["pieces"] <= c["grid"] and c["places"] <= c["room"]
            split += c["split"] > 0
            last += c["split"] > 0 and c["items"] > 512 // hkv
        else:
            unsound += not sound(count(indptr, lens, total, hq, hkv, max_len, trusting=1))
    assert split > 300 and last > 30 and unsound > 10     # the batches reach all of it


@pytest.mark.parametrize("hkv", [1, 8, 512, 513, 1024, 1025, 2048, 65536])
@pytest.mark.parametrize("max_len", [1, 769, 8257, 32768, 2**31 - 1])
def test_room_for_parts_has_room_for_their_records(count, hkv, max_len):
    """The join's grid is of records: with places and no record it would be one of nothing."""
    for bs, total in ((1, 1), (2, 300), (256, 256), (257, 257), (8192, 8192)):
        c = count([0] * bs + [total], [max_len] * bs, total, hkv, hkv, max_len)
        assert (c["room"] == 0) == (c["records"] == 0), (bs, total)
        assert c["records"] * 2 <= c["room"] and sound(c)


def test_lines(count):
    """Batches of more than two rounds are split beyond 8192 tokens, smaller ones beyond 768, and
    of more than 256 requests none."""
    room = lambda bs, max_len, hkv=8: count(range(bs + 1), [1] * bs, bs, 4 * hkv, hkv, max_len)["room"]
    assert room(125, 768) == 0 < room(125, 769) and room(125, 8192) > 0
    assert room(126, 8192) == 0 < room(126, 8193)
    assert room(256, 8193) > 0 == room(257, 2**31 - 1, 1)
