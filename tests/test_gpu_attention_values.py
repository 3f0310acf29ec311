"""What values reach in kvc_packed_attention and kvc_shared_prefix_attention: a
NaN that a query sees makes its output and log-sum NaN, and no other query's;
an output is a weighted mean of V."""
import math

import pytest
import torch

from _attn import attend, bf, check, draw, gen
from _gpu import dev
from test_gpu_packed import _run
from test_gpu_shared_prefix import Case

pytestmark = pytest.mark.gpu

NAN = 0x7FC0
# short and long blocks, and keys cut over workgroups
PACKED = [([40, 129, 1, 700], 8, 2), ([900, 1300, 5], 8, 2), ([2048], 4, 1), ([769] * 24, 32, 8)]
# slots, kv heads of 8 query heads, new tokens: up to 64 rows of a kv head, and more
SHARED = [(3, 2, 1), (8, 1, 1), (4, 2, 4), (9, 1, 1), (33, 2, 1), (12, 2, 7)]


def _nan(x):
    return bf(x).isnan()


# ---------------------------------------------------------------- NaN that a query sees
@pytest.mark.parametrize("lens,hq,hkv", PACKED)
def test_packed_nan_query_and_key(K, lens, hq, hkv):
    g = gen(hq + hkv)
    n = sum(lens)
    q, k, v = draw(g, n, hq, 128), draw(g, n, hkv, 128), draw(g, n, hkv, 128)
    want, want_lse = _run(K, lens, hq, hkv, q, k, v)
    s = max(range(len(lens)), key=lambda i: lens[i])        # the longest sequence: a query, then a key of it
    lo, row = sum(lens[:s]), lens[s] * 2 // 3
    q2 = q.clone()
    q2[lo + row, hq - 1, 5] = NAN
    out, lse = _run(K, lens, hq, hkv, q2, k, v)
    hit = torch.zeros((n, hq), dtype=torch.bool, device=dev())
    hit[lo + row, hq - 1] = True
    assert _nan(out)[hit].all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])
    k2 = k.clone()
    k2[lo + row, hkv - 1, 77] = NAN
    out, lse = _run(K, lens, hq, hkv, q, k2, v)
    hit.zero_()
    hit[lo + row:lo + lens[s], hq - hq // hkv:] = True
    assert _nan(out)[hit].all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])


def _same_but(c, want, hit):
    """hit: [slots, new, query heads], the rows that are NaN; the others have the bits of the case without it."""
    assert _nan(c.out)[hit].all() and c.lse[hit].isnan().all()
    assert torch.equal(c.out[~hit], want.out[~hit]) and torch.equal(c.lse[~hit], want.lse[~hit])


@pytest.mark.parametrize("slots,hkv,n_new", SHARED)
@pytest.mark.parametrize("n_prefix", [0, 2, 3001])
def test_shared_nan_query_and_key(K, slots, hkv, n_new, n_prefix):
    lens = [n_new + 61 * i % 700 for i in range(slots)]
    lens[slots // 2] = 0                                     # an idle slot
    make = lambda: Case(K, n_prefix, lens, n_new, 8, hkv, 16, seed=slots + n_prefix)  # noqa: E731
    want = make().run()
    live = torch.zeros((slots, n_new, 8), dtype=torch.bool, device=dev())
    for s, x in enumerate(lens):
        live[s] = x > 0
    none = torch.zeros_like(live)
    grp = slice(8 - 8 // hkv, 8)                             # the query heads of the last kv head
    # a query
    c, hit = make(), none.clone()
    c.q[slots - 1, n_new - 1, 7, 64] = NAN
    hit[slots - 1, n_new - 1, 7] = True
    _same_but(c.run(), want, hit)
    # a key of the prefix: every query of its head that is in use
    if n_prefix:
        for row in {0, n_prefix - 1, n_prefix // 2}:
            c = make()
            c.kp[row, hkv - 1, 127] = NAN
            hit = none.clone()
            hit[:, :, grp] = live[:, :, grp]
            _same_but(c.run(), want, hit)
    # an own key: the slot's queries from its row on
    s = slots - 1
    for back in {0, n_new - 1, min(n_new, lens[s] - 1)}:
        c, row = make(), lens[s] - 1 - back
        c.k[int(c.table[s, row // 16]), row % 16, hkv - 1, 3] = NAN
        hit = none.clone()
        hit[s, max(n_new - 1 - back, 0):, grp] = True
        _same_but(c.run(), want, hit)


def test_scores_that_leave_float32(K):
    # a score of +inf, like a NaN: the softmax of it is none
    g = gen(3)
    q, k, v = draw(g, 100, 4, 128), draw(g, 100, 2, 128), draw(g, 100, 2, 128)
    q[:, :, 0], k[:, :, 0] = 0, 0
    want, want_lse = _run(K, [100], 4, 2, q, k, v)
    q[60, 3, 0], k[20, 1, 0] = 0x7F00, 0x7F00                # 2^127 each
    hit = torch.zeros((100, 4), dtype=torch.bool, device=dev())
    hit[60, 3] = True
    out, lse = _run(K, [100], 4, 2, q, k, v)
    assert _nan(out)[hit].all() and lse[hit].isnan().all()
    assert torch.equal(out[~hit], want[~hit]) and torch.equal(lse[~hit], want_lse[~hit])
    for slots in (4, 40):
        make = lambda: Case(K, 900, [5 + i for i in range(slots)], 1, 8, 2, 16, seed=slots)  # noqa: E731
        want = make()
        want.q[:, :, :, 0] = 0
        want.kp[:, :, 0] = 0
        want.run()
        c = make()
        c.q[:, :, :, 0] = 0
        c.kp[:, :, 0] = 0
        c.q[1, 0, 2, 0], c.kp[333, 0, 0] = 0x7F00, 0x7F00
        hit = torch.zeros((slots, 1, 8), dtype=torch.bool, device=dev())
        hit[1, 0, 2] = True
        _same_but(c.run(), want, hit)


@pytest.mark.parametrize("slots", [3, 40])
def test_values_that_are_not_finite_reach_their_own_slot_only(K, slots):
    # a later draft token's infinite value has weight zero for earlier ones of its slot, and may spoil them; no other
    lens = [20 + 3 * i for i in range(slots)]
    make = lambda: Case(K, 200, lens, 4, 8, 2, 16, seed=7)  # noqa: E731
    want, c = make().run(), make()
    row = lens[1] - 1
    c.v[int(c.table[1, row // 16]), row % 16] = 0x7F80
    c.run()
    rest = [s for s in range(slots) if s != 1]
    assert torch.equal(c.out[rest], want.out[rest]) and torch.equal(c.lse, want.lse)


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


# ---------------------------------------------------------------- a mean of V
# An output is a weighted mean of V.  A row whose values are all equal has that value as its output, whatever its
# weights: they are rounded to bf16 for the product with V, and so have to be the ones whose sum it is divided by (the
# long kernels' divisor is within 2^-11 of that).  The float32 sums of up to 4,000 weights and of their products with
# one value are off by less than 2^-12 of themselves each; 1.9921875 is 2^-9 from the next value's border, relative to
# itself, so the bits are the same.
SAME = 0x3FFF


@pytest.mark.parametrize("scale", [0.02, 0.0, 0.3])
@pytest.mark.parametrize("lens,hq,hkv", PACKED)
def test_packed_output_of_equal_values(K, lens, hq, hkv, scale):
    g = gen(len(lens) + hq)
    n = sum(lens)
    q, k = draw(g, n, hq, 128, scale=1.5), draw(g, n, hkv, 128, scale=1.5)
    v = torch.full((n, hkv, 128), SAME, dtype=torch.int16, device=dev())
    out, _ = _run(K, lens, hq, hkv, q, k, v, scale)
    assert (out == SAME).all(), int((out != SAME).sum())


@pytest.mark.parametrize("scale", [0.02, 0.0, 0.3])
@pytest.mark.parametrize("slots,hkv,n_new", SHARED)
@pytest.mark.parametrize("n_prefix", [0, 700, 3001])
def test_shared_output_of_equal_values(K, slots, hkv, n_new, n_prefix, scale):
    c = Case(K, n_prefix, [n_new + 37 * i % 600 for i in range(slots)], n_new, 8, hkv, 16, seed=slots)
    c.vp.fill_(SAME)
    c.v.masked_fill_(c.v != NAN, SAME)          # (rows that no slot holds stay NaN)
    c.run(scale)
    assert (c.out == SAME).all(), int((c.out != SAME).sum())


@pytest.mark.parametrize("slots,n_new", [(2, 1), (2, 40)])
def test_shared_output_of_one_dominant_key(K, slots, n_new):
    # own rows of which one has nearly all of the weight, 129.45 times that of an earlier one: between two bf16 values,
    # and too little more for the offset of the exponents to follow
    c = Case(K, 0, [200] * slots, n_new, 8, 1, 16, seed=1)
    c.q.fill_(0)
    c.q[..., 0] = 0x3F80                                     # 1
    c.v.masked_fill_(c.v != NAN, SAME)
    for s in range(slots):
        for row in range(200):
            a = {3: 0.0, 130: 1.0}.get(row, -8.0)
            c.k[int(c.table[s, row // 16]), row % 16] = 0
            c.k[int(c.table[s, row // 16]), row % 16, 0, 0] = torch.tensor(a).to(torch.bfloat16).view(torch.int16).item()
    c.run(math.log(129.45))
    assert (c.out == SAME).all()
    assert (c.lse - math.log(130.45)).abs().max() < 2.0 ** -18 * 5   # each score is one exact product


# ---------------------------------------------------------------- many new tokens
@pytest.mark.parametrize("lens,n_new,hq,hkv,page_rows", [([300, 513, 120], 300, 8, 2, 16), ([700], 600, 4, 1, 8),
                                                         ([1500, 1024], 1024, 2, 1, 64), ([5000], 4096, 2, 1, 64)])
@pytest.mark.parametrize("n_prefix", [0, 333])
def test_question_over_the_context(K, lens, n_new, hq, hkv, page_rows, n_prefix):
    # a question of hundreds of tokens: its rows pass the borders of the own rows' chunks
    Case(K, n_prefix, lens, n_new, hq, hkv, page_rows, seed=n_new).run().check()
