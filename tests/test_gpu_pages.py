"""Page tables on the GPU against the plain model: every entry, every count, every list, every byte."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as k4
from pages_model import Pages
from paper_2605_16928_amd import rtp
from gpu_util import DEV, i32, ws_alloc
from kv4_util import check_row, queries

pytestmark = pytest.mark.gpu


class Both:
    """The model and the device's map, called together and compared after every call."""

    def __init__(self, n_seqs, row, n_pages, page_size):
        self.model = Pages(n_seqs, row, n_pages, page_size)
        self.table = torch.full((n_seqs, row), 77, dtype=torch.int32, device=DEV)
        self.refs = torch.full((n_pages,), 77, dtype=torch.int32, device=DEV)
        self.map = rtp.page_map(self.table, self.refs, page_size)
        self.status = torch.zeros(2, dtype=torch.int32, device=DEV)
        rtp.rtp_kv_pages_init(self.map)
        self.check()

    def check(self, what=""):
        torch.cuda.synchronize()
        np.testing.assert_array_equal(self.table.cpu().numpy(), self.model.table, err_msg=what)
        np.testing.assert_array_equal(self.refs.cpu().numpy(), self.model.refs, err_msg=what)

    def put(self, table=None, refs=None):
        """Sets the state by hand."""
        if table is not None:
            self.model.table[:] = table
            self.table.copy_(torch.from_numpy(self.model.table))
        if refs is not None:
            self.model.refs[:] = refs
            self.refs.copy_(torch.from_numpy(self.model.refs))

    def extend(self, seq, old, new):
        n = len(seq)
        src, dst = (torch.full((n,), -9, dtype=torch.int32, device=DEV) for _ in range(2))
        ws = ws_alloc(rtp.rtp_kv_pages_workspace_bytes(self.map, n))
        ws.fill_(0xff)
        rtp.rtp_kv_pages_extend(self.map, i32(seq), i32(old), i32(new), n, src, dst, self.status, ws)
        pairs, status = self.model.extend(seq, old, new)
        self.check("extend")
        assert list(zip(src.tolist(), dst.tolist())) == pairs
        assert self.status.tolist() == status
        return src, dst, status

    def fork(self, src, dst, n):
        rtp.rtp_kv_pages_fork(self.map, i32(src), i32(dst), i32(n), len(src))
        self.model.fork(src, dst, n)
        self.check("fork")

    def truncate(self, seq, keep):
        rtp.rtp_kv_pages_truncate(self.map, i32(seq), None if keep is None else i32(keep), len(seq))
        self.model.truncate(seq, keep)
        self.check("truncate")

    def compact(self):
        n = len(self.model.refs)
        src, dst = (torch.full((n,), -9, dtype=torch.int32, device=DEV) for _ in range(2))
        ws = ws_alloc(rtp.rtp_kv_pages_workspace_bytes(self.map, 0))
        ws.fill_(0xff)
        rtp.rtp_kv_pages_compact(self.map, src, dst, self.status, ws)
        moves, status = self.model.compact()
        self.check("compact")
        assert self.status.tolist() == status
        assert list(zip(src.tolist(), dst.tolist()))[:len(moves)] == moves
        assert (src[len(moves):] == -9).all() and (dst[len(moves):] == -9).all()
        return src, dst, status


@pytest.mark.parametrize("n_pages,page_size", [(1, 16), (63, 16), (64, 64), (65, 32), (1000, 16), (70000, 16), (200001, 64)])
def test_random_life_of_a_pool(n_pages, page_size):
    """Sequences grow, are forked, cut back, end and move, until pages lack and after: pools of one mask word to four workgroups."""
    print(f"[case] pages, pool of {n_pages}", flush=True)
    rng = np.random.default_rng(n_pages)
    n_seqs, row = 12, max(4, min(n_pages // 3, 2500))
    both = Both(n_seqs, row, n_pages, page_size)
    if n_pages > 65536:                                # most of the pool is taken, so that ranks cross workgroups
        refs = (rng.random(n_pages) < 0.97).astype(np.int32)
        both.put(refs=refs)
    length = [0] * n_seqs
    for step in range(40):
        what = rng.integers(0, 10)
        if what < 5:
            seq = rng.permutation(n_seqs)[:rng.integers(1, n_seqs + 1)].tolist()
            new = [length[b] + int(rng.integers(0, 1 + min(n_pages * page_size // 8, 700 * page_size))) for b in seq]
            new = [min(x, row * page_size) for x in new]
            _, _, status = both.extend(seq, [length[b] for b in seq], new)
            if status[0] == 0:
                for b, x in zip(seq, new):
                    length[b] = x
        elif what < 7:
            a, b = rng.permutation(n_seqs)[:2].tolist()
            both.truncate([b], None)
            n = int(rng.integers(0, length[a] + 1))
            both.fork([a], [b], [n])
            length[b] = n
        elif what < 9:
            seq = rng.permutation(n_seqs)[:3].tolist()
            keep = [int(rng.integers(0, length[b] + 1)) for b in seq]
            both.truncate(seq, keep)
            for b, x in zip(seq, keep):
                length[b] = x
        else:
            both.compact()
    both.compact()


def test_shared_last_pages():
    """A prompt and its forks grow at once: every one whose last page is shared gets its own, full shared pages stay shared, and a
    sequence that does not grow, or whose last page is full, copies nothing."""
    print("[case] pages, shared last pages", flush=True)
    both = Both(6, 8, 40, 16)
    both.extend([0, 1], [0, 0], [40, 32])
    both.fork([0, 0, 0, 1], [2, 3, 4, 5], [40, 40, 20, 32])
    src, dst, _ = both.extend([0, 2, 3, 4, 5], [40, 40, 40, 20, 32], [41, 48, 100, 20, 33])
    assert (src >= 0).tolist() == [True, True, True, False, False]
    both.truncate([2, 2, 3], [0, 0, 5])                # listed twice: released once
    both.extend([4], [20], [21])
    both.compact()
    # cut back into a page that is shared: the next append needs a page of its own again
    both.fork([0], [2], [41])
    both.truncate([0], [20])
    src, _, _ = both.extend([0], [20], [21])
    assert src.tolist() == [int(both.table[2, 1])]


def test_what_does_not_fit_changes_nothing():
    print("[case] pages, shortage", flush=True)
    both = Both(3, 4, 6, 16)
    both.extend([0, 1], [0, 0], [48, 16])
    assert both.extend([0, 1, 2], [48, 16, 0], [64, 17, 16])[2] == [1, 2]        # three wanted, two free
    assert both.extend([2], [0], [65])[2] == [3, 2]                               # (a row of 4: one entry and two pages lack)
    assert both.extend([0], [48], [2 ** 31 - 1])[2][0] > 0
    assert both.extend([0, 2], [48, 0], [64, 16])[2] == [0, 0]
    assert both.extend([1], [16], [16])[2] == [0, 0]
    assert both.extend([1], [16], [17])[2] == [1, 0]
    # ids that are no sequence's, lengths below zero, nothing to do
    assert both.extend([-1, 3, 2 ** 31 - 1, 1], [0, 0, 0, -5], [16, 16, 16, -1])[2] == [0, 0]
    both.fork([-1, 0, 3, 0], [0, 9, 1, 0], [16, 16, 16, 64])
    both.truncate([-1, 3, 5], [0, 0, 0])
    many = 4096
    both.extend([1] + [-1] * (many - 1), [16] * many, [2 ** 31 - 1] * many)
    big = Both(4096, 3, 70000, 16)
    big.extend(list(range(4096)), [0] * 4096, [1 + (7 * i) % 48 for i in range(4096)])
    big.extend(list(range(4096)), [1 + (7 * i) % 48 for i in range(4096)], [2 ** 31 - 1] * 4096)


def test_entries_outside_the_pool():
    """Entries that name no page of the pool are passed over by every call."""
    print("[case] pages, entries outside the pool", flush=True)
    both = Both(4, 5, 10, 16)
    both.put(table=np.array([[0, 10, -7, 3, 2 ** 31 - 1], [1, 2, -1, -1, -1], [-1] * 5, [-1] * 5]), refs=[1, 1, 1, 1] + [0] * 6)
    both.fork([0], [2], [80])
    both.extend([0, 1], [30, 20], [31, 33])
    both.compact()
    both.truncate([0, 2], None)
    both.compact()


@pytest.mark.parametrize("n_pages", [1, 64, 130, 65536, 65537, 140000])
def test_compaction(n_pages):
    print(f"[case] compaction of {n_pages}", flush=True)
    rng = np.random.default_rng(n_pages)
    for share in (0.0, 0.3, 1.0, "front", "back"):
        both = Both(7, 600, n_pages, 16)
        used = np.arange(n_pages) < n_pages // 2 if share == "front" else np.arange(n_pages) >= n_pages // 2 if share == "back" else \
            rng.random(n_pages) < share
        refs = used * rng.integers(1, 4, n_pages)
        ids = np.flatnonzero(used)
        table = np.full((7, 600), -1)
        if len(ids):
            table[:] = rng.choice(ids, (7, 600))
            table[rng.random((7, 600)) < 0.2] = -1
        both.put(table=table, refs=refs)
        both.compact()


def test_copy_moves_the_named_pages_only():
    print("[case] page copies", flush=True)
    rng = np.random.default_rng(1)
    n_pages = 37
    shapes = [(3, n_pages, 16 * 128), (1, n_pages, 16), (5, n_pages, 4096 + 48), (2, n_pages, 64, 128)]
    pools = [torch.from_numpy(rng.integers(0, 256, s, dtype=np.uint8)).to(DEV) for s in shapes]
    pools.append(torch.from_numpy(rng.integers(0, 256, (n_pages, 4, 512), dtype=np.uint8)).to(DEV).transpose(0, 1))   # page-major
    wide = torch.from_numpy(rng.integers(0, 256, (2, n_pages, 96), dtype=np.uint8)).to(DEV)
    pools.append(wide[:, :, 16:64])                    # rows of a wider buffer
    pools.append(torch.randn((2, n_pages, 16, 128), device=DEV).to(torch.bfloat16))
    pools += [torch.from_numpy(rng.integers(0, 256, (1, n_pages, 32), dtype=np.uint8)).to(DEV) for _ in range(60)]    # three launches
    want = [p.clone() for p in pools]
    wide_want = wide.clone()
    src = [5, 5, 36, -1, 3, 37, 7, 2 ** 31 - 1, 11, 12]
    dst = [0, 1, 2, 4, -1, 6, 37, 8, 11, 13]           # pairs outside the pool are passed over, 11 -> 11 changes nothing
    for s, d in list(zip(src, dst))[:9]:
        if 0 <= s < n_pages and 0 <= d < n_pages:
            for w in want:
                w[:, d] = w[:, s]
            wide_want[:, d, 16:64] = wide_want[:, s, 16:64]
    desc = rtp.page_pools(pools)
    rtp.rtp_kv_pages_copy(desc, n_pages, i32(src), i32(dst), len(src), i32([9]))       # the count on the device ends the list
    torch.cuda.synchronize()
    for i, (p, w) in enumerate(zip(pools, want)):
        assert torch.equal(p, w), f"pool {i}"
    assert torch.equal(wide, wide_want)
    for count in (0, -3):
        rtp.rtp_kv_pages_copy(desc, n_pages, i32([5]), i32([9]), 1, i32([count]))
    torch.cuda.synchronize()
    assert all(torch.equal(p, w) for p, w in zip(pools, want))
    rtp.rtp_kv_pages_copy(desc, n_pages, i32([12]), i32([13]), 1, i32([50]))           # (a count beyond n is cut)
    torch.cuda.synchronize()
    assert all(torch.equal(p[:, 13], w[:, 12]) for p, w in zip(pools, want))


@pytest.mark.parametrize("n_pages", [20000, 70001])
def test_thousands_of_requests(n_pages):
    """More requests than threads of a workgroup, in a pool of one and of two: forks that take their own last page among sequences that
    grow by several pages, by none, or are no sequences."""
    print(f"[case] pages, 4000 requests, pool of {n_pages}", flush=True)
    rng = np.random.default_rng(n_pages)
    both = Both(4000, 6, n_pages, 16)
    both.put(refs=(np.arange(n_pages) % 5 == 1).astype(np.int32))        # (others' pages, so that the fresh ones have gaps)
    first = [int(x) for x in rng.integers(1, 33, 1500)]
    both.extend(list(range(1500)), [0] * 1500, first)
    kids = list(range(1500, 3500))
    parents = [int(x) for x in rng.integers(0, 1500, len(kids))]
    both.fork(parents, kids, [first[p] for p in parents])
    old = first + [first[p] for p in parents] + [0] * 500
    seq = rng.permutation(4000).tolist()
    new = [old[b] + int(rng.integers(0, 45)) if b % 7 else old[b] for b in seq]
    src, _, status = both.extend([b if i % 11 else -b - 1 for i, b in enumerate(seq)], [old[b] for b in seq], new)
    assert status[0] == 0 and (src >= 0).sum() > 1024
    both.compact()


def test_copies_that_stream():
    """More than 64 MB in one call, pieces that are not whole, two page sizes, and a list that the device's count cuts short."""
    print("[case] page copies, large", flush=True)
    n_pages, n = 900, 400
    pools = [torch.randint(0, 256, (5, n_pages, 4096 * 9 + 16 * 37), dtype=torch.uint8, device=DEV),
             torch.randint(0, 256, (n_pages, 3, 2048), dtype=torch.uint8, device=DEV).transpose(0, 1)]
    g = torch.Generator().manual_seed(3)
    ids = torch.randperm(n_pages, generator=g)
    src, dst = ids[:n].to(DEV, torch.int32), ids[n:2 * n].to(DEV, torch.int32)
    desc = rtp.page_pools(pools)
    for count in (n - 1, 3):
        want = [p.clone() for p in pools]
        for w, p in zip(want, pools):
            w[:, dst[:count].long()] = p[:, src[:count].long()]
        rtp.rtp_kv_pages_copy(desc, n_pages, src, dst, n, i32([count]))
        torch.cuda.synchronize()
        assert all(torch.equal(p, w) for p, w in zip(pools, want)), count
        for p in pools:
            p.copy_(p.flip(0))                         # (other bytes for the next list)


def test_a_page_that_all_its_holders_leave():
    """The bytes are copied before the page is handed out again; a call whose pages are lacking leaves it shared."""
    print("[case] pages, left by all holders", flush=True)
    both = Both(5, 3, 6, 16)
    pool = torch.randint(0, 256, (2, 6, 64), dtype=torch.uint8, device=DEV)
    old = pool.clone()
    both.extend([0], [0], [20])
    both.fork([0, 0], [1, 2], [20, 20])
    src, dst, status = both.extend([0, 1, 2], [20] * 3, [21] * 3)
    rtp.rtp_kv_pages_copy(rtp.page_pools([pool]), 6, src, dst, 3)
    assert both.refs[1].item() == 0 and status == [0, 1]
    both.extend([3], [0], [17])
    assert both.table[3].tolist() == [1, 5, -1]
    pool[:, 1] = 0                                     # (its new owner writes)
    for p in (2, 3, 4):
        assert torch.equal(pool[:, p], old[:, 1])
    both.truncate([3], None)
    both.fork([0, 0], [3, 4], [20, 20])
    before = both.table.clone(), both.refs.clone()
    assert both.extend([0, 3, 4], [21, 20, 20], [22, 21, 21])[2] == [1, 2]
    assert torch.equal(both.table, before[0]) and torch.equal(both.refs, before[1])
