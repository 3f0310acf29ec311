"""Page tables and page copies (kvc_pages_*) against the oracle, which does
one slot after the other.  Everything is integers or moved bytes: equal, with
no tolerance."""
import numpy as np
import pytest
import torch

import oracle
from _gpu import up, bytes_buf, dev

pytestmark = pytest.mark.gpu


class Pool:
    """A pool on the GPU beside its oracle."""

    def __init__(self, K, n_pages, page_rows, n_slots, max_pages, hkv=1, layers=1, seed=0):
        self.K, self.t = K, oracle.PageTables(n_pages, page_rows, n_slots, max_pages)
        self.ref, self.table, self.len = up(self.t.ref), up(self.t.table), up(self.t.len)
        self.P = K.Pages(n_pages, page_rows, n_slots, max_pages, self.ref, self.table, self.len)
        self.wb = K.kvc_pages_workspace(self.P)
        self.ws = bytes_buf(self.wb)
        self.hkv, self.layers = hkv, layers
        g = torch.Generator(device=dev())
        g.manual_seed(seed)
        shape = (layers, n_pages, page_rows, hkv, 128)
        self.k = torch.randint(-32768, 32767, shape, generator=g, device=dev(), dtype=torch.int16)
        self.v = torch.randint(-32768, 32767, shape, generator=g, device=dev(), dtype=torch.int16)

    def equal(self):
        torch.cuda.synchronize()
        for name in ("ref", "table", "len"):
            assert np.array_equal(getattr(self, name).cpu().numpy(), getattr(self.t, name)), name

    def trim(self, keep):
        self.K.kvc_pages_trim(self.P, up(np.asarray(keep, np.int32)))
        self.t.trim(keep)
        self.equal()

    def fork(self, src):
        self.ws.fill_(0xEE)
        self.K.kvc_pages_fork(self.P, up(np.asarray(src, np.int32)), self.ws, self.wb)
        self.t.fork(src)
        self.equal()

    def reserve(self, n_new, max_new):
        n = len(self.t.len)
        rows = torch.full((n, max_new), -7, dtype=torch.int32, device=dev())
        src, dst, short = (torch.full((m,), -7, dtype=torch.int32, device=dev()) for m in (n, n, 2))
        self.ws.fill_(0xEE)
        self.K.kvc_pages_reserve(self.P, up(np.asarray(n_new, np.int32)), max_new, rows, src, dst, short, self.ws,
                                 self.wb)
        want = self.t.reserve(n_new, max_new)
        self.equal()
        for name, a, b in zip(("rows", "copy_src", "copy_dst", "shortage"), (rows, src, dst, short), want):
            assert np.array_equal(a.cpu().numpy(), b), (name, a.cpu().numpy(), b)
        return rows, src, dst, want[3]

    def compact(self):
        half = len(self.t.ref) // 2
        src, dst, counts = (torch.full((m,), -7, dtype=torch.int32, device=dev()) for m in (half, half, 2))
        self.ws.fill_(0xEE)
        self.K.kvc_pages_compact(self.P, src, dst, counts, self.ws, self.wb)
        want = self.t.compact()
        self.equal()
        for name, a, b in zip(("move_src", "move_dst", "counts"), (src, dst, counts), want):
            assert np.array_equal(a.cpu().numpy(), b), name
        return src, dst, counts

    def copy(self, src, dst, count=None):
        k, v = self.k.clone(), self.v.clone()
        self.K.kvc_pages_copy(self.P, src, dst, src.numel(), count, self.layers, self.hkv, 128, self.k, self.v)
        torch.cuda.synchronize()
        n = src.numel() if count is None else min(src.numel(), max(int(count), 0))
        np_ = len(self.t.ref)
        for a, b in zip(src[:n].tolist(), dst[:n].tolist()):
            if 0 <= a < np_ and 0 <= b < np_:
                k[:, b], v[:, b] = self.k[:, a], self.v[:, a]
        assert torch.equal(self.k, k) and torch.equal(self.v, v)


@pytest.mark.parametrize("page_rows,n_slots,n_pages,max_pages", [(8, 1, 5, 4), (16, 7, 40, 9), (64, 33, 90, 3),
                                                                 (1024, 3, 11, 4), (8, 1500, 6001, 7)])
def test_random_steps(K, page_rows, n_slots, n_pages, max_pages):
    rng = np.random.default_rng(page_rows + n_slots)
    p = Pool(K, n_pages, page_rows, n_slots, max_pages, hkv=1)
    top = max_pages * page_rows
    for step in range(12):
        print(f"pages {page_rows} x {n_pages}, {n_slots} slots, step {step}", flush=True)
        max_new = int(rng.integers(1, 2 * page_rows))
        room = np.maximum(top - p.t.len, 0)
        want = np.minimum(rng.integers(-2, max_new + 3, n_slots), room if step % 4 else top + 1)
        _, src, dst, short = p.reserve(want, max_new)
        p.copy(src, dst)
        keep = np.where(rng.random(n_slots) < 0.3, rng.integers(-1, top + 2, n_slots), -1)
        p.trim(keep)
        fork = np.where(rng.random(n_slots) < 0.3, rng.integers(-3, n_slots + 3, n_slots), -1)
        p.fork(fork)
        if step % 3 == 2:
            src, dst, counts = p.compact()
            p.copy(src, dst, counts[1:])


def test_holders_of_a_shared_page_take_turns(K):
    # one sequence continued by 20: all write, so 20 copies and the last holder keeps the page; if one does not
    # write, every writer gets a copy
    p = Pool(K, 64, 16, 21, 3, hkv=2, layers=3)
    p.reserve([21] + [0] * 20, 32)
    p.fork([0] * 21)
    rows, src, dst, _ = p.reserve([1] * 21, 1)
    assert int((dst >= 0).sum()) == 20 and int(dst[20]) == -1
    p.copy(src, dst)
    q = Pool(K, 64, 16, 21, 3)
    q.reserve([21] + [0] * 20, 32)
    q.fork([0] * 21)
    _, src, dst, _ = q.reserve([1] * 10 + [0] + [1] * 10, 1)
    assert int((dst >= 0).sum()) == 20


def test_slots_exchanged(K):
    # a permutation with a cycle, a self-reference and a chain: all from the tables before the call
    p = Pool(K, 50, 8, 6, 5)
    p.reserve([3, 17, 40, 0, 9, 1], 40)
    p.fork([1, 2, 0, 3, 3, 4])


@pytest.mark.parametrize("want,max_new", [([100, 0, 0], 100), ([65, 0, 0], 80), ([8, 8, 41], 41), ([0, 0, 0], 5)])
def test_shortage_changes_nothing(K, want, max_new):
    # pages missing, a table too small, both, and a call that wants nothing
    p = Pool(K, 6, 8, 3, 8)
    p.reserve([5, 0, 0], 5)
    p.reserve(want, max_new)
    p.reserve([3, 8, 8], 8)


def test_odd_lengths_and_entries(K):
    # lengths beyond the table and below zero count as the nearer end, entries outside the pool for no page
    p = Pool(K, 10, 8, 4, 2)
    p.reserve([16, 9, 0, 1], 16)
    p.len.copy_(torch.tensor([99, 9, -5, 1], dtype=torch.int32))
    p.table[1, 0] = 12
    p.K.kvc_pages_trim(p.P, up(np.array([16, 0, 0, 0], np.int32)))
    torch.cuda.synchronize()
    assert p.len.tolist() == [99, 0, -5, 0]
    ref = p.ref.cpu().numpy()
    # slot 0 keeps its two pages; slot 1's first entry named no page, so page 2 stays counted
    assert ref.tolist() == [1, 1, 1, 0, 0, 0, 0, 0, 0, 0], ref


def test_single_page_pool_and_no_slots(K):
    p = Pool(K, 1, 8, 1, 1)
    p.reserve([8], 8)
    p.compact()
    p.trim([0])
    p.compact()
    q = Pool(K, 9, 8, 0, 0)
    q.compact()
    q.reserve([], 3)


@pytest.mark.parametrize("page_rows,hkv,layers", [(8, 1, 1), (8, 3, 2), (16, 8, 5), (1024, 2, 1)])
def test_copy_skips_bad_pairs(K, page_rows, hkv, layers):
    p = Pool(K, 12, page_rows, 1, 1, hkv=hkv, layers=layers)
    src = up(np.array([0, 3, -1, 12, 5, 0, 7], np.int32))
    dst = up(np.array([1, -2, 4, 6, 12, 2, 8], np.int32))
    p.copy(src, dst)
    p.copy(src, dst, up(np.array([6], np.int32)))
    p.copy(src, dst, up(np.array([-1], np.int32)))
    p.copy(src, dst, up(np.array([1000], np.int32)))


def test_copy_past_4_gib(K):
    # a pool whose byte offsets pass 32 bits: 2,100 pages of 1,024 rows of 8 heads (4.4 GB)
    n, pr, hkv = 2100, 1024, 8
    k = torch.zeros((1, n, pr, hkv, 128), dtype=torch.int16, device=dev())
    v = torch.zeros_like(k)
    k[0, n - 1], v[0, n - 1] = 11, 12
    k[0, n - 2], v[0, n - 2] = 13, 14
    P = K.Pages(n, pr, 0, 0, torch.zeros(n, dtype=torch.int32, device=dev()), None, None)
    K.kvc_pages_copy(P, up(np.array([n - 1, n - 2], np.int32)), up(np.array([0, n - 3], np.int32)), 2, None, 1, hkv,
                     128, k, v)
    torch.cuda.synchronize()
    for x, a, b in ((k, 11, 13), (v, 12, 14)):
        assert (x[0, 0] == a).all() and (x[0, n - 3] == b).all() and (x[0, 1:n - 3] == 0).all()


def test_graph_replays(K):
    # a step captured once: each replay continues from the tables the last one left
    p = Pool(K, 300, 8, 12, 20)
    p.reserve([13] * 12, 13)
    one, src = up(np.ones(12, np.int32)), up(np.array([-1, 0] + [-1] * 10, np.int32))
    rows = torch.empty((12, 1), dtype=torch.int32, device=dev())
    a, b, short = (torch.empty(m, dtype=torch.int32, device=dev()) for m in (12, 12, 2))

    def step():
        K.kvc_pages_fork(p.P, src, p.ws, p.wb)
        K.kvc_pages_reserve(p.P, one, 1, rows, a, b, short, p.ws, p.wb)
        K.kvc_pages_copy(p.P, a, b, 12, None, 1, 1, 128, p.k, p.v)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    p.t.fork(src.tolist())
    p.t.reserve([1] * 12, 1)
    p.equal()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for rep in range(5):
        g.replay()
        torch.randn(1 << 20, device=dev()).sum().item()
        p.t.fork(src.tolist())
        want = p.t.reserve([1] * 12, 1)
        p.equal()
        assert np.array_equal(rows.cpu().numpy(), want[0]), rep
