"""kvc_qkv_norm_rope at the low end of float32: heads whose mean square is
subnormal, with eps 0 and with a subnormal eps.

Bar: that of tests/test_gpu_norm_rope.py, and what subnormals lose.  Each of
the 128 squares, the mean and the mean with eps are off by up to 2^-150 (half
the smallest float32) where they are subnormal: 130 of those against a mean
square of m, 128 m before the division, come to (128 / 128 + 2) 2^-150 / m
relative, and half that after the root."""
import numpy as np
import pytest
import torch

import oracle
from _gpu import up, down_bf16, empty_bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("size", [1e-18, 1.2e-19, 1e-19, 5e-20, 2e-20, 1e-20])
@pytest.mark.parametrize("eps", [0.0, 1e-39])
def test_tiny_heads(K, size, eps):
    rng = np.random.default_rng(int(-np.log10(size) * 100))
    n, hq, hk = 9, 3, 2
    x = rng.standard_normal((n, hq + hk, 128))
    x *= size / np.sqrt((x ** 2).mean(-1, keepdims=True))
    y = oracle.f64_to_bf16(x.reshape(n, -1))
    gq, gk = (oracle.f64_to_bf16(1 + 0.3 * rng.standard_normal(128)) for _ in range(2))
    pos = rng.integers(0, 130000, n).astype(np.int32)
    q, k = empty_bf16(n, hq, 128), empty_bf16(n, hk, 128)
    K.kvc_qkv_norm_rope(up(y), n, hq, hk, 0, 128, up(gq), up(gk), eps, up(pos), 500000.0, q, k, None)
    torch.cuda.synchronize()
    x = oracle.bf16_to_f64(y).reshape(n, hq + hk, 128)
    f = oracle.inv_freq(128, 500000.0)
    eps = float(np.float32(eps))
    lost = 3 * 2.0 ** -150 / (size * size + eps) / 2
    for got, heads, gamma in ((q, x[:, :hq], gq), (k, x[:, hq:], gk)):
        want = oracle.rope_rotate(oracle.rms_norm(heads.reshape(-1, 128), gamma, eps).reshape(heads.shape), pos, f)
        have = torch.from_numpy(down_bf16(got).view(np.int16)).view(torch.bfloat16).double().numpy()
        norm = np.sqrt(want[..., :64] ** 2 + want[..., 64:] ** 2)
        bound = 2.0 ** -8 * np.abs(want) + (2.0 ** -19 + 1.02 * lost) * np.concatenate([norm, norm], -1)
        assert np.all(np.abs(have - want) <= bound), float(np.abs(have - want).max())


@pytest.mark.parametrize("eps,nan", [(1e-39, False), (1.4e-45, False), (0.0, True)])
def test_all_zero_head(K, eps, nan):
    # zero over the root of eps, whatever eps > 0; 0 / 0 with eps = 0, as the formula
    y = np.zeros((2, 256), np.uint16)
    g = oracle.f64_to_bf16(np.ones(128))
    q, k = empty_bf16(2, 1, 128), empty_bf16(2, 1, 128)
    K.kvc_qkv_norm_rope(up(y), 2, 1, 1, 0, 128, up(g), up(g), eps, None, 500000.0, q, k, None)
    torch.cuda.synchronize()
    for t in (q, k):
        x = t.view(torch.bfloat16)
        assert x.isnan().all() if nan else not x.any()
