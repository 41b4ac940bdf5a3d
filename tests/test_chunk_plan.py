"""CPU test of how a batch of new tokens is cut into units: the header the kernels use, compiled for the host."""
import ctypes as C
import os
import random
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_16928_amd", "csrc")
SOURCE = """
#include "chunk_plan.h"
using namespace rtp;
static ChunkShape shape(const int* slot_n, int n_slots, int local, int sink, int window, int cap, int n_cu) {
  ChunkShape s = {};
  int first = 0;
  for (int k = 0; k < n_slots; ++k) {
    s.slot_n[k] = slot_n[k];
    s.slot_first[k] = first;
    first += slot_n[k];
    ++s.cnt[slot_n[k]];
  }
  for (int k = 1; k <= 8; ++k) s.tok[k] = kChunkRows / k;
  s.n_slots = n_slots; s.local = local; s.sink = sink; s.window = window; s.cap = cap; s.n_cu = n_cu;
  return s;
}
// The splits of every sequence; returns the units of cut tiles.
extern "C" long plan(const int* slot_n, int n_slots, int local, int sink, int window, int cap, int n_cu, int B, const int* n, const int* ctx,
                     int* splits, int* tiles) {
  const ChunkShape s = shape(slot_n, n_slots, local, sink, window, cap, n_cu);
  int longest = 1;
  uint64_t work = 0;
  for (int b = 0; b < B; ++b) {
    tiles[b] = chunk_tiles(s, n[b]);
    const int kt = n[b] > 0 ? chunk_key_tiles(s, n[b], ctx[b]) : 1;
    if (n[b] > 0) longest = chunk_max(longest, kt);
    work += (uint64_t)tiles[b] * kt;
  }
  const uint32_t magic = chunk_magic(longest);
  uint32_t best = 0xffffffffu;
  int candidate = 1;
  for (int i = 0; i < kChunkCandidates; ++i) {
    uint64_t units = 0, cut = 0;
    for (int b = 0; b < B; ++b) {
      const int S = chunk_splits(n[b] > 0 ? chunk_key_tiles(s, n[b], ctx[b]) : 1, longest, chunk_candidate(i), magic);
      units += (uint64_t)tiles[b] * S;
      cut += S > 1 ? (uint64_t)tiles[b] * S : 0;
    }
    const uint32_t cost = cut > (uint64_t)cap ? 0xffffffffu : chunk_cost(work, units, cut, n_cu);
    if (cost < best) { best = cost; candidate = chunk_candidate(i); }
  }
  long cut = 0;
  for (int b = 0; b < B; ++b) {
    splits[b] = chunk_splits(n[b] > 0 ? chunk_key_tiles(s, n[b], ctx[b]) : 1, longest, candidate, magic);
    if (splits[b] > 1) cut += (long)tiles[b] * splits[b];
  }
  return cut;
}
extern "C" void unit(const int* slot_n, int n_slots, int n, int S, int r, int* out) {
  const ChunkShape s = shape(slot_n, n_slots, 0, 0, 0, 0, 1);
  const ChunkUnit u = chunk_unit(s, n, S, r);
  int step;
  const int first = chunk_unit_of(s, n, S, u.slot, u.tile, &step);
  out[0] = u.slot; out[1] = u.split; out[2] = u.tile; out[3] = first + u.split * step;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    cxx = shutil.which("g++") or shutil.which("c++")
    assert cxx, "a host C++ compiler is needed"
    d = tmp_path_factory.mktemp("chunk")
    (d / "plan.cpp").write_text(SOURCE)
    so = str(d / "plan.so")
    subprocess.run([cxx, "-std=c++17", "-O2", "-shared", "-fPIC", "-w", "-D__host__=", "-D__device__=", "-D__forceinline__=inline", "-I", CSRC,
                    str(d / "plan.cpp"), "-o", so], check=True)
    L = C.CDLL(so)
    L.plan.restype = C.c_long
    return L


def ints(x):
    return (C.c_int * max(len(x), 1))(*x)


@pytest.mark.parametrize("slots", [[1], [4] * 8, [3, 4, 3, 4], [8], [1] * 16, [7, 5, 6, 2]])
@pytest.mark.parametrize("n,S", [(1, 1), (1, 7), (31, 2), (32, 3), (33, 1), (300, 5), (5000, 1)])
def test_every_unit_once(lib, slots, n, S):
    tiles = [-(-n // (256 // k)) for k in slots]
    seen, out = set(), (C.c_int * 4)()
    for r in range(sum(tiles) * S):
        lib.unit(ints(slots), len(slots), n, S, r, out)
        slot, split, tile, back = out
        assert 0 <= slot < len(slots) and 0 <= split < S and 0 <= tile < tiles[slot] and back == r
        seen.add((slot, split, tile))
    assert len(seen) == sum(tiles) * S


def _plan(lib, slots, new, ctx, local=0, sink=4, window=64, cap=1024, n_cu=256):
    splits, tiles = ints([0] * len(new)), ints([0] * len(new))
    cut = lib.plan(ints(slots), len(slots), local, sink, window, cap, n_cu, len(new), ints(new), ints(ctx), splits, tiles)
    return cut, list(splits)[:len(new)], list(tiles)[:len(new)]


def test_cut_units_stay_inside_the_workspace(lib):
    rng = random.Random(1)
    for _ in range(400):
        B = rng.choice([1, 2, 5, 30, 64])
        slots = [rng.randint(1, 8)] * rng.randint(1, 16)
        new = [rng.choice([0, 1, rng.randint(0, 20), rng.randint(0, 9000)]) for _ in range(B)]
        ctx = [n + rng.choice([0, rng.randint(0, 100), rng.randint(0, 1 << rng.randint(1, 26))]) for n in new]
        cap = rng.choice([0, 1, 17, 1024])
        cut, splits, tiles = _plan(lib, slots, new, ctx, rng.randint(0, 1), cap=cap)
        assert 0 <= cut <= cap and min(splits) >= 1 and max(splits) <= 289
        # the share of the workgroups' numbers that the host counts on
        most = sum(-(-n // (256 // k)) for n in new for k in slots)
        assert sum(tiles) == most


def test_few_rows_fill_the_chip(lib):
    _, splits, tiles = _plan(lib, [4] * 8, [1] * 8, [131072] * 8)
    assert 200 <= sum(s * t for s, t in zip(splits, tiles)) <= 512
    _, splits, tiles = _plan(lib, [1] * 4, [4096], [131072])
    assert sum(s * t for s, t in zip(splits, tiles)) == 256
    _, splits, tiles = _plan(lib, [4] * 8, [4096], [32768])
    assert splits == [1]                                       # 512 tiles are two even rounds
    _, splits, _ = _plan(lib, [4] * 2, [1], [40])
    assert splits == [1]


def test_splits_follow_the_lengths(lib):
    _, splits, _ = _plan(lib, [4] * 2, [1] * 4, [100000, 50000, 1000, 10])
    assert splits[0] >= splits[1] >= splits[2] >= splits[3] == 1 and abs(splits[0] - 2 * splits[1]) <= 2
