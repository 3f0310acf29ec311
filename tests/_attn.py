"""Attention in float64 with what its outputs may be off by, for tests.

The kernels multiply exact bf16 products into float32 scores, keep maximum,
sums and log-sum in float32 and round each weight once to bf16 for the product
with V.  For a row with weights P over values v:

* out: |got - want| <= 2^-8 |want| (its own rounding) + (2^-8 + d) sum_j P_j
  |v_j| (each weight off by half a bf16 step, and by the error d of its
  exponent and of the float32 sums);
* lse: off by d.

d: a score is a float32 sum of 128 products, off by at most 2^-24 (128 + 2)
A, A = scale sum_e |q_e k_e|, once in the weight and once in the maximum or the
sum it is divided by; sums of n positive terms and their joins add at most
2^-24 (n + 64) and exp2, log2 and the final products a few units: 2^-20 (1 +
|lse|) holds those.
"""
import math

import torch


def attend(q, k, v, sees, scale=None):
    """q [r, D], k, v [n, D] float64; row i sees the first sees[i] keys.  out, lse, bounds of both."""
    scale = 1.0 / math.sqrt(q.shape[1]) if not scale else scale
    n = k.shape[0]
    if n == 0:
        z = torch.zeros_like(q)
        return z, torch.full_like(q[:, 0], -math.inf), z, torch.zeros_like(q[:, 0])
    at = torch.arange(n, device=q.device)
    s = (q @ k.T * scale).masked_fill(at >= sees[:, None], -math.inf)
    m = s.max(1).values
    dead = m == -math.inf
    p = torch.exp(s - torch.where(dead, torch.zeros_like(m), m)[:, None])
    z = p.sum(1)
    p = p / torch.where(dead, torch.ones_like(z), z)[:, None]
    out, lse = p @ v, torch.where(dead, m, m + torch.log(z))
    a = (q.abs() @ k.abs().T).max(1).values * scale
    d = 2.0 ** -24 * (260 * a + n + 64) + 2.0 ** -20 * (1 + torch.where(dead, torch.zeros_like(lse), lse.abs()))
    return out, lse, 2.0 ** -8 * out.abs() + (2.0 ** -8 + d)[:, None] * (p @ v.abs()), d


def bf(t):
    """int16 bits on the GPU as float64."""
    return t.view(torch.bfloat16).double()


def draw(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda:0") * scale).to(torch.bfloat16).view(torch.int16)


def gen(seed):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return g


def check(got_out, got_lse, want):
    """Asserts one set of rows: bits of out [r, D], lse [r] or None, attend()'s answer."""
    out, lse, b_out, b_lse = want
    err = (bf(got_out) - out).abs()
    assert bool((err <= b_out + 1e-30).all()), float((err - b_out).max())
    if got_lse is not None:
        dead = torch.isinf(lse)
        assert torch.equal(torch.isneginf(got_lse), dead)
        e = (got_lse.double() - lse)[~dead].abs() - b_lse[~dead]
        assert not e.numel() or float(e.max()) <= 0, float(e.max())
