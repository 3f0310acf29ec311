"""kvc_shared_prefix_attention against float64 attention over prefix and own
rows together (bounds: tests/_attn.py)."""

import numpy as np
import pytest
import torch

from _attn import attend, bf, check, draw, gen
from _gpu import bytes_buf, dev, up

pytestmark = pytest.mark.gpu


class Case:
    """A batch: own rows in randomly placed pages, NaN in every row that no slot holds."""

    def __init__(self, K, n_prefix, lens, n_new, hq, hkv, page_rows, spare=2, seed=0, junk=0x7FC0, max_pages=None):
        g = gen(seed)
        self.K, self.lens, self.n_new, self.hq, self.hkv, self.n = K, lens, n_new, hq, hkv, n_prefix
        b = len(lens)
        have = [-(-x // page_rows) for x in lens]
        mp = max(have + [1]) + 1 if max_pages is None else max_pages
        n_pages = sum(have) + spare
        order = torch.randperm(n_pages, generator=g, device=dev()).to(torch.int32).tolist()
        table = np.full((b, mp), 2 ** 30, dtype=np.int32)       # entries behind the last one mean nothing
        self.k = torch.full((n_pages, page_rows, hkv, 128), junk, dtype=torch.int16, device=dev())
        self.v = self.k.clone()
        self.own = []
        for s, x in enumerate(lens):
            table[s, :have[s]] = [order.pop() for _ in range(have[s])]
            k, v = draw(g, x, hkv, 128, scale=1.5), draw(g, x, hkv, 128)
            at = torch.arange(x, device=dev())
            pg = torch.from_numpy(table[s].astype(np.int64)).to(dev())[at // page_rows]
            self.k[pg, at % page_rows], self.v[pg, at % page_rows] = k, v
            self.own.append((k, v))
        self.kp, self.vp = draw(g, n_prefix, hkv, 128, scale=1.5), draw(g, n_prefix, hkv, 128)
        self.q = draw(g, b, n_new, hq, 128)
        self.table, self.len = up(table), up(np.asarray(lens, np.int32))
        self.P = K.Pages(n_pages, page_rows, b, mp, None, self.table, self.len)
        self.wb = K.kvc_shared_prefix_workspace(self.P, n_prefix, n_new, hq, hkv, 128)
        self.ws = torch.full((max(self.wb, 16),), 0xFF, dtype=torch.uint8, device=dev())
        self.out = torch.full((b, n_new, hq, 128), 0x7FC1, dtype=torch.int16, device=dev())
        self.lse = torch.full((b, n_new, hq), 7.0, device=dev())

    def run(self, scale=0.0, lse=True, stream=None):
        self.K.kvc_shared_prefix_attention(self.q, self.n_new, self.kp if self.n else None, self.vp if self.n else None,
                                           self.n, self.P, self.k, self.v, self.hq, self.hkv, 128, scale, self.out,
                                           self.lse if lse else None, self.ws, self.wb, stream=stream)
        torch.cuda.synchronize()
        return self

    def check(self, scale=0.0, slots=None, gone=()):
        """gone: own rows (slot, row) that are left out."""
        grp = self.hq // self.hkv
        for s in (range(len(self.lens)) if slots is None else slots):
            x = self.lens[s]
            keep = torch.tensor([r for r in range(x) if (s, r) not in gone], dtype=torch.int64, device=dev())
            t = torch.arange(self.n_new, device=dev()) + x - self.n_new
            sees = torch.where(t >= 0, self.n + (keep[None, :] <= t[:, None]).sum(1), torch.zeros_like(t))
            for g in range(self.hkv):
                k = torch.cat([bf(self.kp[:, g]), bf(self.own[s][0][keep, g])])
                v = torch.cat([bf(self.vp[:, g]), bf(self.own[s][1][keep, g])])
                q = bf(self.q[s, :, g * grp:(g + 1) * grp]).reshape(-1, 128)
                want = attend(q, k, v, sees.repeat_interleave(grp), scale)
                check(self.out[s, :, g * grp:(g + 1) * grp].reshape(-1, 128),
                      self.lse[s, :, g * grp:(g + 1) * grp].reshape(-1), want)
        return self


@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 1), (7, 1), (3, 3), (64, 1), (32, 8)])
@pytest.mark.parametrize("n_prefix", [0, 1, 31, 32, 33, 127, 129, 1000])
def test_decode(K, n_prefix, hq, hkv):
    Case(K, n_prefix, [5, 1, 0, 33, 64, 100], 1, hq, hkv, 16, seed=n_prefix + hq).run().check()


@pytest.mark.parametrize("page_rows", [8, 16, 32, 64, 1024])
@pytest.mark.parametrize("n_new", [1, 2, 5, 40])
def test_pages_and_new_tokens(K, page_rows, n_new):
    # slots shorter than the new tokens (padded on the left), at page and tile borders, longer than a chunk
    lens = [0, 1, n_new - 1, n_new, n_new + 1, 31, 32, 33, 511, 512, 513, 700]
    Case(K, 100, lens, n_new, 8, 2, page_rows, seed=page_rows + n_new).run().check()


@pytest.mark.parametrize("slots,n_new,hq,hkv,n_prefix", [(1, 1, 32, 8, 20000), (9, 1, 4, 1, 50001), (17, 3, 28, 4, 4099),
                                                         (64, 1, 32, 8, 3001), (40, 4, 8, 8, 2000), (100, 2, 7, 1, 999),
                                                         (300, 1, 4, 1, 6001), (33, 8, 16, 2, 5003)])
def test_batches(K, slots, n_new, hq, hkv, n_prefix):
    rng = np.random.default_rng(slots)
    lens = [int(x) for x in rng.integers(0, 300, slots)]
    c = Case(K, n_prefix, lens, n_new, hq, hkv, 16, seed=slots).run()
    c.check(slots=sorted({0, 1 % slots, slots // 2, slots - 1}))
    out, lse = c.out.clone(), c.lse.clone()
    c.out.fill_(0)
    c.run(lse=False)
    assert torch.equal(c.out, out) and torch.equal(c.lse, lse)


def test_scale_large_scores_and_dominant_part(K):
    # weights all on one part: the others' log-sums lie hundreds below
    for scale in (0.0, 1.0, 1e-4):
        c = Case(K, 700, [3, 600, 40], 2, 8, 2, 32, seed=3)
        c.kp[300:310] = (c.kp[300:310].view(torch.bfloat16) * 8).view(torch.int16)
        c.run(scale).check(scale)


def test_no_slots_and_table_without_entries(K):
    c = Case(K, 50, [0, 0], 1, 4, 1, 8, max_pages=0)
    c.run()
    assert not c.out.any() and torch.isneginf(c.lse).all()
    K.kvc_shared_prefix_attention(None, 1, None, None, 0, K.Pages(1, 8, 0, 0, None, None, None), None, None, 4, 1, 128,
                                  0.0, None, None, None, 0)


def test_lengths_and_entries_out_of_range(K):
    c = Case(K, 90, [64, 50, 20], 3, 8, 2, 8, seed=4)
    # a page that names nothing: its rows are left out
    c.table[0, 2], c.table[1, 0] = -1, c.P.n_pages
    gone = {(0, r) for r in range(16, 24)} | {(1, r) for r in range(8)}
    c.run().check(gone=gone)
    # the last page too
    c.table[0, 7] = -5
    c.run().check(gone=gone | {(0, r) for r in range(56, 64)})
    # all of a slot's pages
    c.table[2, :3] = 2 ** 30
    c.run().check(gone=gone | {(0, r) for r in range(56, 64)} | {(2, r) for r in range(20)})
    # lengths outside the table count as the nearer end
    d = Case(K, 90, [24, 0], 1, 8, 2, 8, seed=5, max_pages=3)
    d.run()
    want = d.out.clone()
    d.len.copy_(torch.tensor([1000, -7], dtype=torch.int32))
    d.run()
    assert torch.equal(d.out, want)


@pytest.mark.parametrize("junk", [0x7F80, -128, 0x7FFF])
def test_rows_behind_a_length_may_hold_anything(K, junk):
    want = Case(K, 64, [1, 9, 30, 65], 2, 8, 2, 32, seed=6, junk=0).run()
    got = Case(K, 64, [1, 9, 30, 65], 2, 8, 2, 32, seed=6, junk=junk).run()
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)


@pytest.mark.parametrize("slots,hkv", [(4, 2), (40, 2)])
def test_idle_slots_may_hold_anything(K, slots, hkv):
    # NaN and infinite queries in slots that are not in use, beside others in the same 32 rows
    lens = [0 if i % 3 == 1 else 7 + i for i in range(slots)]
    want = Case(K, 150, lens, 1, 8, hkv, 16, seed=12).run()
    got = Case(K, 150, lens, 1, 8, hkv, 16, seed=12)
    for i in range(1, slots, 3):
        got.q[i] = 0x7FC0 if i % 2 else 0x7F80
    got.run()
    assert torch.equal(got.out, want.out) and torch.equal(got.lse, want.lse)
    assert not got.out[1].any() and torch.isneginf(got.lse[1]).all()   # an idle slot: zeros, -inf
    got.check(slots=[0, 2])


def test_pool_past_4_gib(K):
    # pages whose byte offsets pass 32 bits
    n_pages, pr, hkv, hq = 2100, 1024, 8, 16
    k = torch.zeros((n_pages, pr, hkv, 128), dtype=torch.int16, device=dev())
    v = torch.zeros_like(k)
    g = gen(7)
    x, n_prefix = 1500, 77
    table = np.array([[n_pages - 1, n_pages - 2]], np.int32)
    own_k, own_v = draw(g, x, hkv, 128), draw(g, x, hkv, 128)
    for src, dst in ((own_k, k), (own_v, v)):
        dst[n_pages - 1], dst[n_pages - 2, :x - pr] = src[:pr], src[pr:]
    c = Case(K, n_prefix, [10], 1, hq, hkv, 8, seed=7)
    c.P = K.Pages(n_pages, pr, 1, 2, None, up(table), up(np.array([x], np.int32)))
    c.k, c.v, c.lens, c.own = k, v, [x], [(own_k, own_v)]
    c.wb = K.kvc_shared_prefix_workspace(c.P, n_prefix, 1, hq, hkv, 128)
    c.ws = bytes_buf(c.wb)
    c.run().check()


def test_prefix_past_4_gib(K):
    # a prefix of 2.2 million rows of 8 heads: 4.5 GB of keys
    c = Case(K, 2_200_000, [3], 1, 8, 8, 8, seed=8).run()
    c.check()


def test_graph_replays_follow_the_tables(K):
    # captured once; lengths and tables change between replays
    c = Case(K, 333, [40, 50, 60, 0], 1, 8, 2, 16, seed=9)
    c.run()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.kvc_shared_prefix_attention(c.q, 1, c.kp, c.vp, c.n, c.P, c.k, c.v, 8, 2, 128, 0.0, c.out, c.lse, c.ws, c.wb)
    for rep, lens in enumerate(([40, 50, 60, 0], [39, 1, 0, 0], [17, 50, 33, 0], [40, 50, 60, 0])):
        c.len.copy_(torch.tensor(lens, dtype=torch.int32))
        c.lens = lens
        graph.replay()
        torch.randn(1 << 20, device=dev()).sum().item()
        torch.cuda.synchronize()
        saved = c.own
        c.own = [(k[:x], v[:x]) for (k, v), x in zip(saved, lens)]
        c.check()
        c.own = saved


def test_other_stream(K):
    c = Case(K, 2000, [40, 50], 1, 8, 2, 16, seed=10).run()
    want = c.out.clone()
    c.out.fill_(0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    c.run(stream=s)
    assert torch.equal(c.out, want)
