"""kvc_qkv_norm_rope against the oracle's norm and rotation in float64.

Bar: half a bfloat16 step of the exact value (2^-8 of it) plus 2^-19 of the
pair's norm for the float32 work: the sum of 128 squares (19 roundings, halved
by the root), root, division, two products, sine and cosine (2^-22 for the
reduced angle held in float32) and the rotation's two roundings come to less
than 20 x 2^-24 of the pair's norm."""
import numpy as np
import pytest
import torch

import oracle
from _gpu import up, down_bf16, empty_bf16

pytestmark = pytest.mark.gpu


def _want(y, pos, hq, hk, hv, gq, gk, eps, f):
    n = y.shape[0]
    x = oracle.bf16_to_f64(y).reshape(n, hq + hk + hv, 128)
    q = oracle.rms_norm(x[:, :hq].reshape(-1, 128), gq, eps).reshape(n, hq, 128)
    k = oracle.rms_norm(x[:, hq:hq + hk].reshape(-1, 128), gk, eps).reshape(n, hk, 128)
    return oracle.rope_rotate(q, pos, f), oracle.rope_rotate(k, pos, f)


def _close(bits, want):
    got = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16).double().numpy()
    norm = np.sqrt(want[..., :64] ** 2 + want[..., 64:] ** 2)
    bound = 2.0 ** -8 * np.abs(want) + 2.0 ** -19 * np.concatenate([norm, norm], -1)
    return bool(np.all(np.abs(got - want) <= bound))


@pytest.mark.parametrize("hq,hk,hv,n", [(32, 8, 8, 37), (28, 4, 4, 5), (1, 1, 1, 1), (0, 8, 0, 9), (5, 0, 3, 66),
                                        (3, 2, 0, 2), (40, 40, 0, 11), (8, 2, 2, 1000)])
@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_norm_rope(K, hq, hk, hv, n, eps):
    rng = np.random.default_rng(hq + 3 * hk + n)
    y = oracle.f64_to_bf16(rng.standard_normal((n, (hq + hk + hv) * 128)) * np.exp(rng.standard_normal((n, 1)) * 3))
    gq, gk = (oracle.f64_to_bf16(1 + 0.3 * rng.standard_normal(128)) for _ in range(2))
    pos = rng.integers(0, 130000, n).astype(np.int32)
    f = oracle.inv_freq(128, 500000.0)
    q, k, v = (empty_bf16(n, max(h, 1), 128) for h in (hq, hk, hv))
    K.kvc_qkv_norm_rope(up(y), n, hq, hk, hv, 128, up(gq) if hq else None, up(gk) if hk else None, eps, up(pos),
                        500000.0, q if hq else None, k if hk else None, v if hv else None)
    torch.cuda.synchronize()
    wq, wk = _want(y, pos, hq, hk, hv, gq, gk, eps, f)
    assert not hq or _close(down_bf16(q), wq)
    assert not hk or _close(down_bf16(k), wk)
    if hv:
        assert np.array_equal(down_bf16(v), y.reshape(n, -1, 128)[:, hq + hk:])


def test_implicit_positions_frequency_table_and_zero_heads(K):
    rng = np.random.default_rng(3)
    n, hq, hk = 70, 2, 2
    yf = rng.standard_normal((n, (hq + hk) * 128))
    yf[4, :128] = 0.0                                    # an all-zero head stays zero with eps > 0
    y = oracle.f64_to_bf16(yf)
    g = oracle.f64_to_bf16(rng.standard_normal(128))
    f = 0.5 ** np.arange(64)
    q, k = empty_bf16(n, hq, 128), empty_bf16(n, hk, 128)
    K.kvc_qkv_norm_rope(up(y), n, hq, hk, 0, 128, up(g), up(g), 1e-6, None, 0.0, q, k, None, inv_freq=list(f))
    torch.cuda.synchronize()
    wq, wk = _want(y, np.arange(n), hq, hk, 0, g, g, 1e-6, f)
    assert _close(down_bf16(q), wq) and _close(down_bf16(k), wk)
    assert not (down_bf16(q)[4, 0] & 0x7FFF).any()


def test_values_whose_squares_leave_float32(K):
    # squares up to 1e36 sum to a finite float32; a tiny head keeps its norm
    rng = np.random.default_rng(4)
    y = oracle.f64_to_bf16(np.concatenate([rng.standard_normal((3, 128)) * 1e17, rng.standard_normal((3, 128)) * 1e-12]))
    g = oracle.f64_to_bf16(np.ones(128))
    q = empty_bf16(6, 1, 128)
    K.kvc_qkv_norm_rope(up(y), 6, 1, 0, 0, 128, up(g), None, 0.0, None, 500000.0, q, None, None)
    torch.cuda.synchronize()
    wq, _ = _want(y, np.arange(6), 1, 0, 0, g, g, 0.0, oracle.inv_freq(128, 500000.0))
    assert _close(down_bf16(q), wq)


@pytest.mark.parametrize("hq,hk", [(3, 0), (0, 3), (0, 0)])
def test_weights_that_no_head_uses_are_not_looked_at(K, hq, hk):
    # (a pointer of theirs need not be aligned, nor hold 128 weights, nor be apart from the outputs)
    rng = np.random.default_rng(5)
    n, hv = 4, 2
    y = oracle.f64_to_bf16(rng.standard_normal((n, (hq + hk + hv) * 128)))
    g = oracle.f64_to_bf16(1 + 0.3 * rng.standard_normal(128))
    q, k, v = (empty_bf16(n, max(h, 1), 128) for h in (hq, hk, hv))
    other = v.view(-1)[1:]
    K.kvc_qkv_norm_rope(up(y), n, hq, hk, hv, 128, up(g) if hq else other, up(g) if hk else other, 1e-5, None,
                        500000.0, q if hq else None, k if hk else None, v)
    torch.cuda.synchronize()
    wq, wk = _want(y, np.arange(n), hq, hk, hv, g, g, 1e-5, oracle.inv_freq(128, 500000.0))
    assert not hq or _close(down_bf16(q), wq)
    assert not hk or _close(down_bf16(k), wk)
    assert np.array_equal(down_bf16(v), y.reshape(n, -1, 128)[:, hq + hk:])
