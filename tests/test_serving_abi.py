"""Refusals and host logic of the packed attention, the head norms, the pages
and the attention over a shared prefix (no GPU needed: every invalid argument
is refused before any HIP call; the addresses are fake and never used)."""
import pytest

A = 1 << 44                       # fake device addresses, far apart
STEP = 1 << 40


def _status(fn, *a, **kw):
    import paper_2609_09768_amd as K
    try:
        fn(*a, **kw)
    except K.KvcError as e:
        return e.status, str(e)
    return 0, ""


def _no_gpu():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: valid calls on fake addresses are not made")


# ---------------------------------------------------------------- packed sequences
def _packed(K, pack, **kw):
    a = dict(pack=pack, plan=K.Plan(A, 1 << 30, 0), q=A + STEP, k=A + 2 * STEP, v=A + 3 * STEP, n_rows=100,
             softmax_scale=0.0, out=A + 4 * STEP, lse=A + 5 * STEP, ws=A + 6 * STEP, ws_bytes=1 << 40)
    a.update(kw)
    return _status(K.kvc_packed_attention, **a)


def _pack_plan(K, pack, nbytes=None):
    """A plan descriptor as kvc_pack_plan_upload would fill it: the id comes back in the refusal of a wrong one."""
    st, msg = _packed(K, pack, plan=K.Plan(A, 1 << 30, 2), n_rows=max(pack.n_rows, 1))
    assert st == K.KVC_ERR_INVALID_ARG and "other sequences" in msg, msg
    pid = int(msg.split("these ")[1].split(")")[0], 16)
    return K.Plan(A, K.kvc_pack_plan_bytes(pack) if nbytes is None else nbytes, pid)


def test_pack_validation(K):
    bad, uns = K.KVC_ERR_INVALID_ARG, K.KVC_ERR_UNSUPPORTED
    assert _status(K.kvc_pack_plan_bytes, None)[0] == bad
    assert _status(K.kvc_pack_plan_bytes, K.Pack([3, -1], 8, 2))[0] == bad
    assert _status(K.kvc_pack_plan_bytes, K.Pack([3], 6, 4))[0] == bad
    assert _status(K.kvc_pack_plan_bytes, K.Pack([3], 8, 0))[0] == bad
    assert _status(K.kvc_pack_plan_bytes, K.Pack([3], 8, 2, 64))[0] == uns
    assert _status(K.kvc_pack_plan_bytes, K.Pack([2**31 - 1, 2**31 - 1], 1, 1))[0] == bad
    st, msg = _status(K.kvc_pack_plan_bytes, K.Pack([2**30], 64, 8))
    assert st == bad and "one launch" in msg
    for lens in ([], [0], [0, 0, 5], [1] * 1000, [124000]):
        assert K.kvc_pack_plan_bytes(K.Pack(lens, 8, 2)) > 0
        assert K.kvc_packed_attention_workspace(K.Pack(lens, 8, 2)) >= 0


def test_packed_attention_refusals(K):
    bad, wsp = K.KVC_ERR_INVALID_ARG, K.KVC_ERR_WORKSPACE
    pack = K.Pack([60, 40], 8, 2)
    plan = _pack_plan(K, pack)
    assert _packed(K, pack, plan=None)[0] == bad
    assert _packed(K, pack, plan=K.Plan(A + 4, 1 << 30, plan.layout_id))[0] == bad
    assert _packed(K, pack, plan=K.Plan(A, K.kvc_pack_plan_bytes(pack) - 1, plan.layout_id))[0] == wsp
    for other in (K.Pack([40, 60], 8, 2), K.Pack([100], 8, 2), K.Pack([60, 40], 8, 4), K.Pack([60, 40], 4, 2)):
        assert _packed(K, other, plan=plan)[0] == bad
    # the plan of a chunked request is no plan of packed sequences
    L = K.Layout([60, 40], 0, 8, 2)
    assert _packed(K, pack, plan=K.Plan(A, 1 << 30, K.kvc_layout_id(L)))[0] == bad
    assert _packed(K, pack, plan=plan, n_rows=99)[0] == bad
    assert _packed(K, pack, plan=plan, n_rows=2**31)[0] == bad
    for scale in (-1.0, float("nan"), float("inf")):
        assert _packed(K, pack, plan=plan, softmax_scale=scale)[0] == bad
    for name in ("q", "k", "v", "out"):
        assert _packed(K, pack, plan=plan, **{name: None})[0] == bad
        assert _packed(K, pack, plan=plan, **{name: A + 8 * STEP + 8})[0] == bad
    assert _packed(K, pack, plan=plan, lse=A + 5 * STEP + 2)[0] == bad
    for name in ("q", "k", "v", "lse"):
        st, msg = _packed(K, pack, plan=plan, **{name: A + 4 * STEP + 1024})
        assert st == bad and "overlaps" in msg, name
    st, msg = _packed(K, pack, plan=K.Plan(A + 4 * STEP, 1 << 20, plan.layout_id))
    assert st == bad and "plan" in msg
    # one long sequence is cut and needs its workspace
    one = K.Pack([2048], 4, 1)
    need = K.kvc_packed_attention_workspace(one)
    assert need > 0
    p1 = _pack_plan(K, one)
    assert _packed(K, one, plan=p1, n_rows=2048, ws=None, ws_bytes=need)[0] == bad
    assert _packed(K, one, plan=p1, n_rows=2048, ws=A + 6 * STEP + 8)[0] == bad
    assert _packed(K, one, plan=p1, n_rows=2048, ws_bytes=need - 1)[0] == wsp


def test_packed_attention_without_rows_and_valid_calls(K):
    for lens in ([], [0, 0]):
        K.kvc_packed_attention(K.Pack(lens, 8, 2), None, None, None, None, 0, 0.0, None, None)
    _no_gpu()
    pack = K.Pack([60, 40], 8, 2)
    st, _ = _packed(K, pack, plan=_pack_plan(K, pack))
    assert st == K.KVC_ERR_DEVICE
    assert _status(K.kvc_pack_plan_upload, pack, A, K.kvc_pack_plan_bytes(pack))[0] == K.KVC_ERR_DEVICE
    assert _status(K.kvc_pack_plan_upload, pack, A, K.kvc_pack_plan_bytes(pack) - 1)[0] == K.KVC_ERR_WORKSPACE
    assert _status(K.kvc_pack_plan_upload, pack, A + 4, 1 << 30)[0] == K.KVC_ERR_INVALID_ARG


@pytest.mark.parametrize("lens,hq,hkv", [([1], 1, 1), ([2048], 4, 1), ([5, 0, 700, 33], 7, 1), ([1000] * 30, 32, 8),
                                         ([9000, 3], 28, 4), ([31, 32, 33, 64, 65], 16, 2)])
def test_plan_image_covers_every_tile_once(K, lens, hq, hkv):
    # the image built into a caller's staging memory: header (24 bytes), work items of eight int32 from byte 256,
    # joins behind them.  Every unit's key tiles are covered exactly once, parts are numbered once, longest first.
    import torch
    import numpy as np
    pack = K.Pack(lens, hq, hkv)
    nb = K.kvc_pack_plan_bytes(pack)
    if torch.cuda.is_available():
        pytest.skip("the upload would go to a fake address")
    img = np.zeros(nb, np.uint8)
    assert _status(K.kvc_pack_plan_upload, pack, A, nb, staging=img.ctypes.data)[0] == K.KVC_ERR_DEVICE
    n_long, n_short, n_joins, n_parts = img[8:24].view(np.int32)
    n_items = n_long + n_short
    items = img[256:256 + 32 * n_items].view(np.int32).reshape(n_items, 8)
    j0 = 256 + (32 * n_items + 255) // 256 * 256
    joins = img[j0:j0 + 32 * n_joins].view(np.int32).reshape(n_joins, 8)
    assert (items[:n_long, 1] > 768).all() and (items[n_long:, 1] <= 768).all()
    assert (np.diff(items[:n_long, 4]) <= 0).all()
    # the short sequences' queues: two workgroups a CU, none empty, loads (tiles and two per block) nearly even
    queues = min(int(n_short), 512 // hkv)
    q0 = j0 + (32 * n_joins + 255) // 256 * 256
    start = img[q0:q0 + 4 * (queues + 1)].view(np.int32)
    assert nb >= q0 + 4 * (queues + 1) and start[0] == 0 and start[-1] == n_short and (np.diff(start) > 0).all()
    load = [int((items[n_long + a:n_long + b, 4] + 2).sum()) for a, b in zip(start[:-1], start[1:])]
    assert not load or max(load) - min(load) <= 10
    grp, row0, seen = hq // hkv, 0, 0
    parts = {}
    for r, n, b, t0, nt, part in items[:, :6]:
        parts.setdefault((int(r), int(n), int(b)), []).append((int(t0), int(nt), int(part)))
    for n in lens:
        units, wide = -(-n // 32) * grp, 8 if n > 768 else 4
        for b in range(-(-units // wide)):
            last = min(32 * ((wide * b + wide - 1) // grp + 1), n) - 1
            got = sorted(parts.pop((row0, n, b)))
            at = 0
            for t0, nt, part in got:
                assert t0 == at and nt > 0 and (part >= 0) == (len(got) > 1)
                at += nt
            assert at == last // 64 + 1
            if len(got) > 1:
                j = [x for x in joins if x[0] == row0 and x[2] == b and x[1] == n]
                assert len(j) == 1 and j[0][4] == len(got) and [p for _, _, p in got] == list(
                    range(j[0][3], j[0][3] + len(got)))
                seen += len(got)
        row0 += n
    assert not parts and seen == n_parts


# ---------------------------------------------------------------- head norms
def test_qkv_norm_rope_refusals(K):
    bad = K.KVC_ERR_INVALID_ARG
    base = dict(y=A, n=10, n_q_heads=4, n_k_heads=2, n_v_heads=2, head_dim=128, gamma_q=A + 5 * STEP,
                gamma_k=A + 6 * STEP, eps=1e-5, pos=A + STEP, rope_theta=1e4, q=A + 2 * STEP, k=A + 3 * STEP,
                v=A + 4 * STEP)
    for kw in (dict(n=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(gamma_q=None), dict(gamma_k=None),
               dict(gamma_q=A + 5 * STEP + 2), dict(y=None), dict(q=None), dict(k=A + 3 * STEP + 4), dict(pos=A + STEP + 1),
               dict(rope_theta=0.0), dict(n_q_heads=-1), dict(gamma_k=A + 2 * STEP + 256), dict(v=A + 3 * STEP),
               dict(inv_freq=[float("nan")] * 64), dict(n_q_heads=1000, n_k_heads=100)):
        assert _status(K.kvc_qkv_norm_rope, **{**base, **kw})[0] == bad, kw
    assert _status(K.kvc_qkv_norm_rope, **{**base, "head_dim": 64})[0] == K.KVC_ERR_UNSUPPORTED
    K.kvc_qkv_norm_rope(**{**base, "n": 0, "y": None})
    _no_gpu()
    for kw in ({}, dict(n_q_heads=0, gamma_q=None, q=None), dict(n_k_heads=0, gamma_k=None, k=None), dict(pos=None)):
        assert _status(K.kvc_qkv_norm_rope, **{**base, **kw})[0] == K.KVC_ERR_DEVICE, kw


# ---------------------------------------------------------------- pages
def _pages(K, **kw):
    a = dict(n_pages=100, page_rows=16, n_slots=8, max_pages=20, ref=A, table=A + STEP, len=A + 2 * STEP)
    a.update(kw)
    return K.Pages(**a)


def _calls(K, P, ws=A + 3 * STEP, wb=1 << 40):
    h = A + 4 * STEP
    return {"trim": lambda: _status(K.kvc_pages_trim, P, h),
            "fork": lambda: _status(K.kvc_pages_fork, P, h, ws, wb),
            "reserve": lambda: _status(K.kvc_pages_reserve, P, h, 4, h + STEP, h + 2 * STEP, h + 3 * STEP, h + 4 * STEP,
                                       ws, wb),
            "compact": lambda: _status(K.kvc_pages_compact, P, h, h + STEP, h + 2 * STEP, ws, wb)}


def test_pages_validation(K):
    bad, uns = K.KVC_ERR_INVALID_ARG, K.KVC_ERR_UNSUPPORTED
    wrong = [(dict(n_pages=0), bad), (dict(n_slots=-1), bad), (dict(max_pages=-1), bad), (dict(page_rows=4), uns),
             (dict(page_rows=24), uns), (dict(page_rows=2048), uns), (dict(page_rows=0), uns), (dict(page_rows=-16), uns),
             (dict(n_pages=2**28), bad), (dict(max_pages=2**27), bad), (dict(n_slots=65537), bad),
             (dict(n_slots=65536, max_pages=2**15), bad), (dict(ref=None), bad), (dict(table=None), bad),
             (dict(len=None), bad), (dict(ref=A + 2), bad), (dict(table=A + STEP + 1), bad), (dict(len=A + 2 * STEP + 3), bad)]
    for kw, want in wrong:
        assert _status(K.kvc_pages_workspace, _pages(K, **kw))[0] == want, kw
        for name, call in _calls(K, _pages(K, **kw)).items():
            assert call()[0] == want, (kw, name)
    assert _status(K.kvc_pages_workspace, None)[0] == bad
    assert K.kvc_pages_workspace(_pages(K)) > 0


def test_pages_refusals(K):
    bad, wsp = K.KVC_ERR_INVALID_ARG, K.KVC_ERR_WORKSPACE
    P, h = _pages(K), A + 4 * STEP
    wb = K.kvc_pages_workspace(P)
    ws = A + 3 * STEP
    for name in ("fork", "reserve", "compact"):
        assert _calls(K, P, ws=None)[name]()[0] == bad
        assert _calls(K, P, ws=ws + 4)[name]()[0] == bad
        assert _calls(K, P, wb=wb - 1)[name]()[0] == wsp
        st, msg = _calls(K, P, ws=A + STEP, wb=wb)[name]()
        assert st == bad and "overlaps" in msg
    assert _status(K.kvc_pages_trim, P, None)[0] == bad
    assert _status(K.kvc_pages_trim, P, h + 1)[0] == bad
    assert _status(K.kvc_pages_trim, P, A + 2 * STEP)[0] == bad           # keep over len
    assert _status(K.kvc_pages_fork, P, None, ws, wb)[0] == bad
    r = dict(pages=P, n_new=h, max_new=4, rows=h + STEP, copy_src=h + 2 * STEP, copy_dst=h + 3 * STEP,
             shortage=h + 4 * STEP, ws=ws, ws_bytes=wb)
    for kw in (dict(max_new=0), dict(max_new=2**29), dict(n_new=None), dict(rows=None), dict(copy_src=None),
               dict(copy_dst=h + 3 * STEP + 2), dict(shortage=None), dict(rows=h), dict(copy_src=h + 3 * STEP + 4)):
        assert _status(K.kvc_pages_reserve, **{**r, **kw})[0] == bad, kw
    c = dict(pages=P, move_src=h, move_dst=h + STEP, counts=h + 2 * STEP, ws=ws, ws_bytes=wb)
    for kw in (dict(move_src=None), dict(move_dst=None), dict(counts=None), dict(counts=h + 2 * STEP + 2), dict(move_dst=h)):
        assert _status(K.kvc_pages_compact, **{**c, **kw})[0] == bad, kw
    y = dict(pages=P, src=h, dst=h + STEP, n_pairs=5, count=h + 2 * STEP, n_layers=2, n_kv_heads=8, head_dim=128,
             k_pages=h + 3 * STEP, v_pages=h + 4 * STEP)
    for kw in (dict(n_pairs=-1), dict(n_layers=-1), dict(n_kv_heads=0), dict(n_kv_heads=65), dict(src=None), dict(dst=None),
               dict(k_pages=None), dict(v_pages=h + 4 * STEP + 8), dict(count=h + 1), dict(v_pages=h + 3 * STEP + 4096),
               dict(src=h + 3 * STEP)):
        assert _status(K.kvc_pages_copy, **{**y, **kw})[0] == bad, kw
    assert _status(K.kvc_pages_copy, **{**y, "head_dim": 64})[0] == K.KVC_ERR_UNSUPPORTED
    K.kvc_pages_copy(**{**y, "n_pairs": 0})
    K.kvc_pages_copy(**{**y, "n_layers": 0})
    empty = _pages(K, n_slots=0, max_pages=0, table=None, len=None)
    K.kvc_pages_trim(empty, None)
    K.kvc_pages_fork(empty, None, None, 0)
    _no_gpu()
    for name, call in _calls(K, P).items():
        assert call()[0] == K.KVC_ERR_DEVICE, name
    assert _status(K.kvc_pages_copy, **y)[0] == K.KVC_ERR_DEVICE
    # copying needs no tables
    assert _status(K.kvc_pages_copy, **{**y, "pages": _pages(K, ref=None)})[0] == K.KVC_ERR_DEVICE


# ---------------------------------------------------------------- attention over a shared prefix
def test_shared_prefix_refusals(K):
    bad, uns, wsp = K.KVC_ERR_INVALID_ARG, K.KVC_ERR_UNSUPPORTED, K.KVC_ERR_WORKSPACE
    P = _pages(K, ref=None)
    need = K.kvc_shared_prefix_workspace(P, 1000, 2, 8, 2, 128)
    assert need > 0
    h = A + 4 * STEP
    base = dict(q=h, n_new=2, k_prefix=h + STEP, v_prefix=h + 2 * STEP, n_prefix=1000, pages=P, k_pages=h + 3 * STEP,
                v_pages=h + 4 * STEP, n_q_heads=8, n_kv_heads=2, head_dim=128, softmax_scale=0.0, out=h + 5 * STEP,
                lse=h + 6 * STEP, ws=h + 7 * STEP, ws_bytes=need)
    call = lambda **kw: _status(K.kvc_shared_prefix_attention, **{**base, **kw})  # noqa: E731
    for kw in (dict(n_new=0), dict(n_new=5000), dict(n_prefix=-1), dict(n_prefix=2**31), dict(pages=None), dict(n_q_heads=7),
               dict(softmax_scale=-0.5), dict(softmax_scale=float("nan")), dict(q=None), dict(out=None), dict(k_prefix=None),
               dict(v_prefix=h + 2 * STEP + 8), dict(k_pages=None), dict(v_pages=h + 8), dict(lse=h + 6 * STEP + 2),
               dict(ws=None), dict(ws=h + 7 * STEP + 8), dict(out=h + 3 * STEP), dict(lse=h + STEP + 64),
               dict(ws=A + STEP), dict(out=A + 2 * STEP)):
        assert call(**kw)[0] == bad, kw
    assert call(head_dim=64)[0] == uns
    assert call(pages=_pages(K, ref=None, page_rows=12))[0] == uns
    assert call(ws_bytes=need - 1)[0] == wsp
    big = _pages(K, n_slots=65536, max_pages=1, ref=None)
    assert _status(K.kvc_shared_prefix_workspace, big, 10, 64, 32, 8, 128)[0] == bad
    K.kvc_shared_prefix_attention(**{**base, "pages": _pages(K, n_slots=0, max_pages=0, ref=None, table=None, len=None),
                                     "q": None})
    _no_gpu()
    assert call()[0] == K.KVC_ERR_DEVICE
    assert call(n_prefix=0, k_prefix=None, v_prefix=None)[0] == K.KVC_ERR_DEVICE
    assert call(lse=None)[0] == K.KVC_ERR_DEVICE


def test_shared_prefix_workspace_holds_every_part(K):
    # at the borders of what a launch takes, and with a table of millions of rows
    for n_slots, max_pages, pr, n_prefix, n_new in ((1, 1, 8, 0, 1), (1, 2**20, 8, 2**31 - 128, 1), (3, 2**17, 1024, 5, 7),
                                                    (65536, 4, 8, 100, 1), (256, 8, 16, 124256, 8)):
        P = _pages(K, n_slots=n_slots, max_pages=max_pages, page_rows=pr, ref=None)
        rows = n_slots * n_new * 4
        assert K.kvc_shared_prefix_workspace(P, n_prefix, n_new, 4, 1, 128) >= (n_prefix > 0) * rows * 129 * 4
