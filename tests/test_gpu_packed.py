"""kvc_packed_attention against float64 attention of each sequence alone
(bounds: tests/_attn.py)."""

import pytest
import torch

from _attn import attend, bf, check, draw, gen
from _gpu import bytes_buf, dev, empty_bf16

pytestmark = pytest.mark.gpu


def _plan(K, lens, hq, hkv):
    pack = K.Pack(lens, hq, hkv)
    pb = K.kvc_pack_plan_bytes(pack)
    return pack, K.kvc_pack_plan_upload(pack, bytes_buf(pb), pb)


def _run(K, lens, hq, hkv, q, k, v, scale=0.0, lse=True):
    n = q.shape[0]
    pack, plan = _plan(K, lens, hq, hkv)
    out = torch.full((n, hq, 128), 0x7FC1, dtype=torch.int16, device=dev())       # NaN bits: left where not written
    ls = torch.full((n, hq), 7.0, device=dev()) if lse else None
    wb = K.kvc_packed_attention_workspace(pack)
    ws = torch.full((max(wb, 16),), 0xFF, dtype=torch.uint8, device=dev())        # NaN partials
    K.kvc_packed_attention(pack, plan, q, k, v, n, scale, out, ls, ws if wb else None, wb)
    torch.cuda.synchronize()
    return out, ls


def _check(lens, hq, hkv, q, k, v, out, lse, scale=0.0, heads=None):
    lo = 0
    for L in lens:
        for h in (range(hq) if heads is None else heads):
            g = h // (hq // hkv)
            for i in range(lo, lo + L, 2048):
                j = min(i + 2048, lo + L)
                want = attend(bf(q[i:j, h]), bf(k[lo:j, g]), bf(v[lo:j, g]),
                              torch.arange(i - lo + 1, j - lo + 1, device=dev()), scale)
                check(out[i:j, h], None if lse is None else lse[i:j, h], want)
        lo += L
    # rows behind the last sequence are left as they were
    assert (out[lo:] == 0x7FC1).all() and (lse is None or (lse[lo:] == 7.0).all())


LENS = [[1], [2, 1, 1], [31, 32, 33], [63, 64, 65, 0, 128, 129], [0, 0], [0, 5, 0], [257], [700, 3, 90], [1] * 70]


@pytest.mark.parametrize("hq,hkv", [(8, 2), (4, 1), (7, 1), (3, 3), (32, 8), (16, 1), (10, 2)])
@pytest.mark.parametrize("lens", LENS, ids=lambda x: "-".join(map(str, x[:6])))
def test_lengths_and_heads(K, lens, hq, hkv):
    g = gen(sum(lens) + hq)
    n = sum(lens) + 3
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128, scale=1.5), draw(g, n, hkv, 128)
    out, lse = _run(K, lens, hq, hkv, q, k, v)
    _check(lens, hq, hkv, q, k, v, out, lse)


# few long sequences: their keys are cut over workgroups and joined (5,000
# rows of 28 heads fill the GPU without that)
@pytest.mark.parametrize("lens,hq,hkv,cut", [([2048], 4, 1, True), ([1500, 1], 1, 1, True),
                                             ([3000, 40, 2000], 8, 2, True), ([5000], 28, 4, False),
                                             ([1025], 9, 3, False), ([1400], 9, 3, True)])
def test_cut_keys(K, lens, hq, hkv, cut):
    g = gen(sum(lens))
    n = sum(lens)
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128, scale=2.0), draw(g, n, hkv, 128)
    assert (K.kvc_packed_attention_workspace(K.Pack(lens, hq, hkv)) > 0) == cut
    out, lse = _run(K, lens, hq, hkv, q, k, v)
    _check(lens, hq, hkv, q, k, v, out, lse, heads=sorted({0, hq // 2, hq - 1}))
    again, _ = _run(K, lens, hq, hkv, q, k, v, lse=False)
    assert torch.equal(out, again)


def test_uncut_batch_matches_the_sparse_entry_point_closely(K):
    # one sequence is causal attention of every row
    g = gen(5)
    n, hq, hkv = 4096, 32, 8
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    out, lse = _run(K, [n], hq, hkv, q, k, v)
    _check([n], hq, hkv, q, k, v, out, lse, heads=[0, 13, 31])


def test_scale_and_large_scores(K):
    # scores up to hundreds, rising along the sequence: the running offset has to move
    g = gen(6)
    lens, hq, hkv = [600, 300], 4, 2
    n = sum(lens)
    ramp = torch.linspace(0.1, 6.0, n, device=dev())[:, None, None]
    q, v = draw(g, n, hq, 128, scale=2.0), draw(g, n, hkv, 128)
    k = (torch.randn((n, hkv, 128), generator=g, device=dev()) * ramp).to(torch.bfloat16).view(torch.int16)
    for scale in (0.0, 0.5, 1e-3):
        out, lse = _run(K, lens, hq, hkv, q, k, v, scale)
        _check(lens, hq, hkv, q, k, v, out, lse, scale)


def test_other_rows_do_not_reach_a_sequence(K):
    # NaN and infinities in the rows of the next sequence and behind the last one
    g = gen(7)
    lens, hq, hkv = [70, 45, 33], 8, 2
    n = sum(lens) + 50
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    want, _ = _run(K, lens, hq, hkv, q, k, v)
    for bits in (0x7FC0, 0x7F80, -128):
        for lo, hi in ((70, 115), (148, n)):
            k2, v2, q2 = k.clone(), v.clone(), q.clone()
            k2[lo:hi], v2[lo:hi], q2[lo:hi] = bits, bits, bits
            got, _ = _run(K, lens, hq, hkv, q2, k2, v2)
            keep = torch.ones(n, dtype=torch.bool, device=dev())
            keep[lo:hi] = False
            assert torch.equal(got[keep], want[keep])


def test_long_batch_past_2g_elements(K):
    # 70,000 rows of 256 query heads: more than 2^31 elements of q and out
    hq, hkv = 256, 1
    lens = [64] * 1000 + [3000, 3000]
    n = sum(lens)
    g = gen(8)
    q = torch.empty((n, hq, 128), dtype=torch.int16, device=dev())
    for i in range(0, n, 10000):
        q[i:i + 10000] = draw(g, *q[i:i + 10000].shape)
    assert q.numel() > 2 ** 31
    k, v = draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    out, lse = _run(K, lens, hq, hkv, q, k, v)
    lo = sum(lens[:-1])
    for h in (0, 255):
        want = attend(bf(q[lo:, h]), bf(k[lo:, 0]), bf(v[lo:, 0]), torch.arange(1, lens[-1] + 1, device=dev()))
        check(out[lo:, h], lse[lo:, h], want)


def test_other_stream_and_graph(K):
    g = gen(9)
    lens, hq, hkv = [900, 17, 1200], 8, 2
    n = sum(lens)
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    want, want_lse = _run(K, lens, hq, hkv, q, k, v)
    pack, plan = _plan(K, lens, hq, hkv)
    wb = K.kvc_packed_attention_workspace(pack)
    out, lse, ws = empty_bf16(n, hq, 128), torch.empty((n, hq), device=dev()), bytes_buf(wb)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    K.kvc_packed_attention(pack, plan, q, k, v, n, 0.0, out, lse, ws, wb, stream=s)
    s.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        K.kvc_packed_attention(pack, plan, q, k, v, n, 0.0, out, lse, ws, wb)
    for rep in range(4):
        out.fill_(0), lse.fill_(0)
        graph.replay()
        torch.randn(1 << 20, device=dev()).sum().item()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse), rep
    # staging memory of the caller: the plan is copied without a wait
    pb = K.kvc_pack_plan_bytes(pack)
    staged = K.kvc_pack_plan_upload(pack, bytes_buf(pb), pb, staging=torch.empty(pb, dtype=torch.uint8, pin_memory=True))
    out.fill_(0)
    K.kvc_packed_attention(pack, staged, q, k, v, n, 0.0, out, None, ws, wb)
    torch.cuda.synchronize()
    assert torch.equal(out, want)
