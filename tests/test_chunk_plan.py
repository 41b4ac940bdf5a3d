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
static ChunkShape shape(const int* members, int n_kv, int group, int local, int sink, int window, int cap, int places) {
  ChunkShape s = {};
  s.group = group; s.n_kv = n_kv; s.local = local; s.sink = sink; s.window = window; s.cap = cap; s.places = (float)places;
  for (int k = 0; k < n_kv; ++k) {
    s.served[k * group / 32] |= (uint32_t)members[k] << (k * group % 32);
    const int n = chunk_bits(members[k]);
    s.n_served += n;
    if (n) { ++s.count[n - 1]; ++s.kv_served; }
  }
  for (int h = 1; h <= 8; ++h) s.per_tile[h - 1] = chunk_inverse(chunk_tokens(0, h));
  for (int h = 8; h >= 1; --h) if (s.count[h - 1]) s.per_most = s.per_tile[h - 1];
  return s;
}
extern "C" void range_of(int n, int k, int S, int* out) { chunk_range(n, k, S, out, out + 1); }
extern "C" int tiles_of(int n, int h, int fine) { return chunk_query_tiles(n, chunk_inverse(chunk_tokens(fine, h))); }
extern "C" int tokens_of(int h, int fine) { return chunk_tokens(fine, h); }
// The splits of every sequence; returns the units of cut tiles.
extern "C" long plan(const int* members, int n_kv, int group, int local, int sink, int window, int cap, int places, int B, const int* n, const int* ctx,
                     int* splits, int* tiles) {
  const ChunkShape s = shape(members, n_kv, group, local, sink, window, cap, places);
  int longest = 1;
  float work = 0;
  for (int b = 0; b < B; ++b) {
    tiles[b] = chunk_tiles(s, n[b]);
    const int kt = n[b] > 0 ? chunk_key_tiles(s, n[b], ctx[b]) : 1;
    if (n[b] > 0) longest = chunk_max(longest, kt);
    work += (float)tiles[b] * (float)kt;
  }
  const uint32_t magic = chunk_magic(longest);
  float best = INFINITY;
  int candidate = 1;
  for (int i = 0; i < kChunkCandidates; ++i) {
    ChunkSums sums = {};
    for (int b = 0; b < B; ++b) {
      const int kt = n[b] > 0 ? chunk_key_tiles(s, n[b], ctx[b]) : 1;
      chunk_sum(&sums, tiles[b], n[b] * s.n_served, kt, chunk_splits(kt, longest, chunk_candidate(i), magic), 1.f / places);
    }
    const float cost = sums.cut_units > (float)cap ? INFINITY : chunk_cost(work, sums, longest, chunk_candidate(i), (float)places);
    if (cost < best) { best = cost; candidate = chunk_candidate(i); }
  }
  long cut = 0;
  for (int b = 0; b < B; ++b) {
    splits[b] = chunk_splits(n[b] > 0 ? chunk_key_tiles(s, n[b], ctx[b]) : 1, longest, candidate, magic);
    if (splits[b] > 1) cut += (long)tiles[b] * splits[b];
  }
  return cut;
}
extern "C" void unit(const int* members, int n_kv, int group, int n, int S, int r, int run_shift, int* out) {
  ChunkShape s = shape(members, n_kv, group, 0, 0, 0, 0, 1);
  s.run_shift = run_shift;
  const ChunkUnit u = chunk_unit(s, n, S, r);
  out[0] = u.kv; out[1] = u.split; out[2] = u.tile; out[3] = u.heads; out[4] = u.tiles; out[5] = u.before; out[6] = u.step;
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


TOKENS = [0, 256, 128, 85, 64, 51, 42, 36, 32]          # per tile, by the number of served heads
MEMBERS = [([1], 1), ([15] * 8, 4), ([7, 15, 0, 13], 4), ([255], 8), ([1] * 16, 1), ([127, 31, 62, 3], 8), ([0, 2, 0, 1], 2)]


@pytest.mark.parametrize("members,group", MEMBERS)
@pytest.mark.parametrize("n,S", [(1, 1), (1, 7), (31, 2), (32, 3), (33, 1), (300, 5), (5000, 1)])
@pytest.mark.parametrize("run_shift", [0, 1, 4])
def test_every_unit_once(lib, members, group, n, S, run_shift):
    heads = [bin(m).count("1") for m in members]
    tiles = [-(-n // TOKENS[h]) if h else 0 for h in heads]
    units, steps, numbers, out = [], [], set(), (C.c_int * 7)()
    for r in range(sum(tiles) * S):
        lib.unit(ints(members), len(members), group, n, S, r, run_shift, out)
        kv, split, tile, h, mine, before, step = out
        assert 0 <= split < S and 0 <= tile < tiles[kv] and h == heads[kv] and mine == tiles[kv] and before == sum(tiles[:kv])
        units.append((kv, split, tile))
        steps.append(step)
        if split == 0:                                  # every tile has a number of its own
            numbers.add(before + mine - 1 - tile)
    assert len(set(units)) == sum(tiles) * S and numbers == set(range(sum(tiles)))
    for r, (kv, split, tile) in enumerate(units):
        if split == 0:                                  # the ranges of a tile are as far apart as the unit says
            assert [units[r + s * steps[r]] for s in range(S)] == [(kv, s, tile) for s in range(S)]
    groups = min(t for t in tiles if t) >> run_shift    # whole groups: those of later tiles first, of every KV head in turn
    if groups > 1:
        block, served = S << run_shift, [kv for kv, t in enumerate(tiles) if t]
        for j in range(groups * len(served)):
            g, kv = j // len(served), served[j % len(served)]
            mine = {(kv, s, tiles[kv] - 1 - (g << run_shift) - k) for s in range(S) for k in range(1 << run_shift)}
            assert set(units[j * block:(j + 1) * block]) == mine


@pytest.mark.parametrize("fine", [0, 3])
@pytest.mark.parametrize("h", range(1, 9))
def test_tiles(lib, h, fine):
    tok, rows = TOKENS[h] if fine == 0 else 32 // h, 256 >> fine
    assert lib.tokens_of(h, fine) == tok and h * tok <= rows < h * (tok + 1)
    rng = random.Random(h)
    for n in list(range(2000)) + [rng.randint(0, 1 << 24) for _ in range(5000)] + [(1 << 24) - k for k in range(600)] + [(1 << 24) // tok * tok + k for k in (-1, 0, 1)]:
        assert lib.tiles_of(n, h, fine) == -(-n // tok)


def _plan(lib, heads, new, ctx, local=0, sink=4, window=64, cap=1024, places=256):
    splits, tiles = ints([0] * len(new)), ints([0] * len(new))
    members = [(1 << h) - 1 for h in heads]
    cut = lib.plan(ints(members), len(heads), 8, local, sink, window, cap, places, len(new), ints(new), ints(ctx), splits, tiles)
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
        most = sum(-(-n // TOKENS[k]) for n in new for k in slots)
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


def test_ranges_are_neighbours_and_alike(lib):
    rng, out = random.Random(2), (C.c_int * 2)()
    for n, S in [(0, 1), (0, 7), (3, 7), (7, 7), (8, 7), (1 << 24, 289)] + [(rng.randint(0, 5000), rng.randint(1, 289)) for _ in range(300)]:
        at = 0
        for k in range(S):
            lib.range_of(n, k, S, out)
            assert out[0] == at and n // S <= out[1] - out[0] <= n // S + 1
            at = out[1]
        assert at == n
