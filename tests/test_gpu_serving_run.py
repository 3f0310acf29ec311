"""The operators around the blended context together, as a request uses them:
chunks prefilled in one packed batch, their caches blended into a context
(the framework's own path), then a batch of sequences that fork, grow and
attend over the context, through two decoding steps."""
import numpy as np
import pytest
import torch

import oracle
from _attn import attend, bf, check, draw, gen
from _gpu import bytes_buf, dev, down_bf16, empty_bf16, up

pytestmark = pytest.mark.gpu

HQ, HKV, D, THETA, EPS = 8, 2, 128, 500000.0, 1e-5


def _split(K, y, pos, gq, gk):
    n = y.shape[0]
    q, k, v = empty_bf16(n, HQ, D), empty_bf16(n, HKV, D), empty_bf16(n, HKV, D)
    K.kvc_qkv_norm_rope(y, n, HQ, HKV, HKV, D, gq, gk, EPS, pos, THETA, q, k, v)
    return q, k, v


def test_chunks_to_answers(K):
    g = gen(11)
    heads = (HQ + 2 * HKV) * D
    gq, gk = (up(oracle.f64_to_bf16(1 + 0.2 * np.random.default_rng(s).standard_normal(D))) for s in (1, 2))

    # 1. three chunks prefilled on their own, positions from 0 in each
    lens = [300, 77, 130]
    n = sum(lens)
    y = draw(g, n, heads)
    local = up(np.concatenate([np.arange(x) for x in lens]).astype(np.int32))
    q, k_src, v_src = _split(K, y, local, gq, gk)
    pack = K.Pack(lens, HQ, HKV)
    pb = K.kvc_pack_plan_bytes(pack)
    plan = K.kvc_pack_plan_upload(pack, bytes_buf(pb), pb)
    wb = K.kvc_packed_attention_workspace(pack)
    out = empty_bf16(n, HQ, D)
    K.kvc_packed_attention(pack, plan, q, k_src, v_src, n, 0.0, out, None, bytes_buf(wb), wb)
    lo = 0
    for x in lens:
        for h in (0, HQ - 1):
            grp = h // (HQ // HKV)
            check(out[lo:lo + x, h], None, attend(bf(q[lo:lo + x, h]), bf(k_src[lo:lo + x, grp]),
                                                  bf(v_src[lo:lo + x, grp]), torch.arange(1, x + 1, device=dev())))
        lo += x

    # 2. the context: the chunks' caches moved to their places, a check layer selects and recomputes
    n_query = 19
    N = n + n_query
    L = K.Layout(lens, n_query, HQ, HKV, D, THETA)
    yq = torch.cat([y, draw(g, n_query, heads)])
    qf, kf, vf = _split(K, yq, up(np.arange(N, dtype=np.int32)), gq, gk)
    pb = K.kvc_plan_bytes(L)
    lplan = K.kvc_plan_upload(L, bytes_buf(pb), pb)
    k_cache, v_cache = empty_bf16(N, HKV, D), torch.cat([v_src, torch.zeros_like(vf[n:])])
    n_sel = K.kvc_recompute_count(0.15, n) + n_query
    sel = torch.empty(n_sel, dtype=torch.int32, device=dev())
    wb = K.kvc_blend_workspace(L)
    K.kvc_blend_prefill_layer(L, lplan, 1, 0.15, k_src, k_cache, v_cache, qf, kf, vf, sel, n_sel,
                              empty_bf16(n_sel, HQ, D), None, bytes_buf(wb), wb)
    # every key stands at its place in the context: the moved ones next to the fresh ones (no cross-attention between
    # chunks enters these keys, so both are the same values up to two roundings)
    a, b = bf(k_cache), bf(kf)
    assert float((a - b).norm() / b.norm()) < 2 * 2.0 ** -8

    # 3. six sequences over the context, of which four start as copies of the first
    slots, pr, pages = 6, 8, 40
    ref, table, length = (torch.zeros(s, dtype=torch.int32, device=dev()) for s in ((pages,), (slots, 5), (slots,)))
    P = K.Pages(pages, pr, slots, 5, ref, table, length)
    kt, vt = (torch.full((pages, pr, HKV, D), 0x7FC0, dtype=torch.int16, device=dev()) for _ in range(2))
    pw = K.kvc_pages_workspace(P)
    pws = bytes_buf(pw)
    copy_src, copy_dst = (torch.empty(slots, dtype=torch.int32, device=dev()) for _ in range(2))
    short = torch.empty(2, dtype=torch.int32, device=dev())
    mirror = oracle.PageTables(pages, pr, slots, 5)
    mirror.table[:] = 0
    own = [[] for _ in range(slots)]                          # (key, value) rows of every sequence

    def grow(n_new, max_new):
        """New tokens of every slot: rows reserved, shared pages copied, keys and values written; then attention."""
        rows = torch.empty((slots, max_new), dtype=torch.int32, device=dev())
        K.kvc_pages_reserve(P, up(np.asarray(n_new, np.int32)), max_new, rows, copy_src, copy_dst, short, pws, pw)
        want = mirror.reserve(n_new, max_new)
        K.kvc_pages_copy(P, copy_src, copy_dst, slots, None, 1, HKV, D, kt, vt)
        pos = np.asarray([[N + len(own[s]) + t for t in range(max_new)] for s in range(slots)], np.int32)
        qn, kn, vn = _split(K, draw(g, slots * max_new, heads), up(pos.reshape(-1)), gq, gk)
        K.kvc_scatter_rows(rows, slots * max_new, 1, kn, vn, slots * max_new, kt, vt, pages * pr, HKV, D)
        assert np.array_equal(rows.cpu().numpy(), want[0]) and not short.any()
        for s in range(slots):
            own[s] += [(kn[s * max_new + t], vn[s * max_new + t]) for t in range(n_new[s])]
        wb = K.kvc_shared_prefix_workspace(P, N, max_new, HQ, HKV, D)
        o, lse = empty_bf16(slots, max_new, HQ, D), torch.empty((slots, max_new, HQ), device=dev())
        # the last max_new rows of a slot are its queries; a shorter slot's first queries have no place (zeros)
        qs = qn.view(slots, max_new, HQ, D)
        K.kvc_shared_prefix_attention(qs, max_new, k_cache, v_cache, N, P, kt, vt, HQ, HKV, D, 0.0, o, lse,
                                      bytes_buf(wb), wb)
        torch.cuda.synchronize()
        for s in range(slots):
            x = len(own[s])
            assert x == int(length[s])
            t = torch.arange(max_new, device=dev()) + x - max_new
            for h in (0, HQ - 1):
                grp = h // (HQ // HKV)
                ko = [bf(k[grp])[None] for k, _ in own[s]]
                vo = [bf(v[grp])[None] for _, v in own[s]]
                k = torch.cat([bf(k_cache[:, grp])] + ko)
                v = torch.cat([bf(v_cache[:, grp])] + vo)
                sees = torch.where(t >= 0, N + t + 1, torch.zeros_like(t))
                check(o[s, :, h], lse[s, :, h], attend(bf(qs[s, :, h]), k, v, sees))

    def tables_equal():
        torch.cuda.synchronize()
        assert np.array_equal(ref.cpu().numpy(), mirror.ref) and np.array_equal(length.cpu().numpy(), mirror.len)
        for s in range(slots):
            held = mirror.held(s)
            assert table[s, :len(held)].tolist() == held

    grow([13, 2, 0, 0, 0, 0], 13)                             # two questions
    src = [-1, -1, 0, 0, 0, 0]
    K.kvc_pages_fork(P, up(np.asarray(src, np.int32)), pws, pw)
    mirror.fork(src)
    for s in range(2, 6):
        own[s] = list(own[0])
    grow([1] * 6, 1)                                          # a token each: shared pages are copied
    keep = [-1, 0, 11, -1, -1, 0]                             # two end, one takes rows back
    K.kvc_pages_trim(P, up(np.asarray(keep, np.int32)))
    mirror.trim(keep)
    own = [x[:kp] if kp >= 0 else x for x, kp in zip(own, keep)]
    move = [torch.empty(pages // 2, dtype=torch.int32, device=dev()) for _ in range(2)]
    counts = torch.empty(2, dtype=torch.int32, device=dev())
    K.kvc_pages_compact(P, move[0], move[1], counts, pws, pw)
    mirror.compact()
    K.kvc_pages_copy(P, move[0], move[1], pages // 2, counts[1:], 1, HKV, D, kt, vt)
    tables_equal()
    grow([1, 0, 3, 2, 3, 0], 3)                               # several tokens, idle slots among them
    tables_equal()
