"""kvc_packed_attention: short sequences whose offsets pass 2^31 elements, the
largest batch of them, and the answers beside those of kvc_sparse_query_attention."""
import pytest
import torch

from _attn import attend, bf, check, draw, gen
from _gpu import bytes_buf, dev, empty_bf16
from test_gpu_packed import _plan, _run

pytestmark = pytest.mark.gpu


def test_short_sequences_past_2g_elements(K):
    # 70,764 rows of 256 query heads; the last two sequences start behind 2^31 elements of q and out
    hq, hkv = 256, 1
    lens = [64] * 1000 + [3000, 3000] + [64, 700]
    n = sum(lens)
    g = gen(8)
    q = torch.empty((n, hq, 128), dtype=torch.int16, device=dev())
    for i in range(0, n, 10000):
        q[i:i + 10000] = draw(g, *q[i:i + 10000].shape)
    k, v = draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    out, lse = _run(K, lens, hq, hkv, q, k, v)
    assert (n - 764) * hq * 128 > 2 ** 31
    start = [0]
    for x in lens:
        start.append(start[-1] + x)
    for s in (0, 517, 999, 1000, 1002, 1003):
        lo, x = start[s], lens[s]
        for h in (0, 101, 255):
            want = attend(bf(q[lo:lo + x, h]), bf(k[lo:lo + x, 0]), bf(v[lo:lo + x, 0]), torch.arange(1, x + 1, device=dev()))
            check(out[lo:lo + x, h], lse[lo:lo + x, h], want)


def test_as_many_short_sequences_as_a_call_takes(K):
    # 65,536 sequences of one row and 512/64 heads: 2^22 blocks of eight units.  A row alone has its v as its output.
    n, hq, hkv = 65536, 512, 64
    g = gen(11)
    q = torch.empty((n, hq, 128), dtype=torch.int16, device=dev())
    for i in range(0, n, 4096):
        q[i:i + 4096] = draw(g, 4096, hq, 128)
    k, v = draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    pack, plan = _plan(K, [1] * n, hq, hkv)
    out, lse = torch.full_like(q, 0x7FC1), torch.full((n, hq), 7.0, device=dev())
    assert K.kvc_packed_attention_workspace(pack) == 0
    K.kvc_packed_attention(pack, plan, q, k, v, n, 0.0, out, lse)
    torch.cuda.synchronize()
    for i in range(0, n, 8192):
        assert torch.equal(out[i:i + 8192].view(-1, hkv, hq // hkv, 128), v[i:i + 8192, :, None].expand(-1, -1, hq // hkv, -1))
    for i in (0, 1, 30000, n - 1):
        for h in (0, 77, 511):
            want = attend(bf(q[i:i + 1, h]), bf(k[i:i + 1, h // 8]), bf(v[i:i + 1, h // 8]), torch.ones(1, device=dev()))
            check(out[i:i + 1, h], lse[i:i + 1, h], want)


@pytest.mark.parametrize("n,hq,hkv", [(4096, 32, 8), (700, 8, 2), (1500, 4, 1)])
def test_one_sequence_beside_the_sparse_entry_point(K, n, hq, hkv):
    # one sequence is kvc_sparse_query_attention with every row selected.  Either divides weights rounded to bf16 (each
    # off by 2^-8 of itself at most) by their own sum, whose relative error is a mean of theirs: 2 x 2^-8 of sum P |v|
    # and d, and 2^-8 of the output for its rounding, which is less than twice attend()'s bound.
    g = gen(5)
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    out, _ = _run(K, [n], hq, hkv, q, k, v)
    pos = torch.arange(n, dtype=torch.int32, device=dev())
    other = empty_bf16(n, hq, 128)
    wb = K.kvc_attention_workspace(n, hq, hkv, 128)
    K.kvc_sparse_query_attention(q, n, None, pos, n, k, v, n, hq, hkv, 128, 0.0, other, None, bytes_buf(wb), wb)
    torch.cuda.synchronize()
    for h in (0, hq // 2, hq - 1):
        want, _, bound, _ = attend(bf(q[:, h]), bf(k[:, h // (hq // hkv)]), bf(v[:, h // (hq // hkv)]),
                                   torch.arange(1, n + 1, device=dev()))
        for a in (out, other):
            assert ((bf(a[:, h]) - want).abs() <= 2 * bound).all()
        assert ((bf(out[:, h]) - bf(other[:, h])).abs() <= 4 * bound).all()
