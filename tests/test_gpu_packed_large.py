"""kvc_packed_attention: the largest batch of short sequences that a call takes."""
import pytest
import torch

from _attn import attend, bf, check, draw, gen
from _gpu import dev
from test_gpu_packed import _plan

pytestmark = pytest.mark.gpu


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
