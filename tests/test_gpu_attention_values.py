"""What values that are not finite reach in kvc_packed_attention and
kvc_shared_prefix_attention."""
import pytest
import torch

from _attn import attend, bf, check, draw, gen
from _gpu import dev
from test_gpu_packed import _run

pytestmark = pytest.mark.gpu


def test_keys_whose_scores_are_all_infinitely_negative(K):
    # weights of zero: the keys that are left answer, and a row of no others has none
    g = gen(4)
    q, k, v = draw(g, 200, 4, 128), draw(g, 200, 2, 128), draw(g, 200, 2, 128)
    q[:, :, 0] = 0x7F00
    k[:, :, 0] = 0
    k[:70, 1, 0] = -256                                      # 0xFF00, -2^127: the first tile's scores and a few more
    out, lse = _run(K, [200], 4, 2, q, k, v)
    assert torch.isneginf(lse[:70, 2:]).all() and not out[:70, 2:].any()
    for h in (2, 3):
        for i in (70, 71, 133, 199):
            want = attend(bf(q[i:i + 1, h]), bf(k[70:i + 1, 1]), bf(v[70:i + 1, 1]), torch.tensor([i - 69], device=dev()))
            check(out[i:i + 1, h], lse[i:i + 1, h], want)
    for h in (0, 1):
        want = attend(bf(q[:, h]), bf(k[:, 0]), bf(v[:, 0]), torch.arange(1, 201, device=dev()))
        check(out[:, h], lse[:, h], want)
