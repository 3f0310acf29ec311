"""The operators around the blended context whose speed matters: what they compute, and on which sizes.

A request's context is blended out of chunks.  Before that, each chunk's cache
was computed by prefilling the chunk on its own, many of them packed into one
batch; afterwards a batch of sequences answers over the one context, each with
rows of its own in the pages of a pool.  Kinds of case:

* ``pack``: ``kvc_packed_attention``, causal attention inside each of many
  packed sequences;
* ``norm``: ``kvc_qkv_norm_rope``, the split of the fused Q/K/V projection with
  an RMS norm of each query and key head before the rotation;
* ``shared``: ``kvc_shared_prefix_attention``, the new tokens of a batch of
  sequences over the shared context and over their own pages;
* ``step``: ``kvc_pages_trim``, ``_fork``, ``_reserve`` and ``_copy``, the page
  tables of one serving step: sequences that end or roll back, slots that
  continue another's sequence, rows for the new tokens, shared pages copied
  before they are written;
* ``compact``: ``kvc_pages_compact`` and ``_copy``, a scattered pool's live
  pages moved to its low end.

``own`` says whether ``run`` takes the library's entry points or the plain
form of the same operator.
"""
import math
import random

import torch

own = False

D = 128
THETA = 500000.0
EPS = 1e-5
DEV = "cuda:0"
BF = torch.bfloat16
INF = float("inf")

# query heads, kv heads
MODELS = {
    "small": (8, 2),
    "llama8b": (32, 8),
    "qwen7b": (28, 4),
    "llama8b-tp8": (4, 1),
    "equal": (8, 8),
}


def listed():
    return [
        # a few short snippets cached together, one of a single token: the time of a launch
        {"name": "pack-snippets-small", "kind": "pack", "model": "small", "lens": "mixed", "seqs": 5, "rows": 161},
        # retrieval documents of 16 to 512 tokens, cached in one batch
        {"name": "pack-32k-docs", "kind": "pack", "model": "llama8b", "lens": "docs", "seqs": 180, "rows": 32000},
        # sequences from a few tokens to thousands, seven query heads to a kv head
        {"name": "pack-20k-mixed-qwen", "kind": "pack", "model": "qwen7b", "lens": "mixed", "seqs": 23, "rows": 20011},
        # the 16 chunks of the 124k-token context
        {"name": "pack-124k", "kind": "pack", "model": "llama8b", "lens": "even", "seqs": 16, "rows": 124000},
        # the new tokens of a small batch
        {"name": "norm-33", "kind": "norm", "model": "llama8b", "rows": 33},
        # the rows selected out of the 124k-token context
        {"name": "norm-18k", "kind": "norm", "model": "llama8b", "rows": 18856},
        # three sequences over a short context
        {"name": "shared-1k-small", "kind": "shared", "model": "small", "prefix": 1088, "slots": 3, "new": 1,
         "tail": 40, "page": 16},
        # a batch over a retrieval context
        {"name": "shared-32k-b16", "kind": "shared", "model": "llama8b", "prefix": 32256, "slots": 16, "new": 1,
         "tail": 300, "page": 32},
        # a few sequences with several draft tokens each, seven query heads to a kv head
        {"name": "shared-61k-b6-new5-qwen", "kind": "shared", "model": "qwen7b", "prefix": 61001, "slots": 6, "new": 5,
         "tail": 700, "page": 64},
        # a large batch over the 124k-token context
        {"name": "shared-124k-b64", "kind": "shared", "model": "llama8b", "prefix": 124256, "slots": 64, "new": 1,
         "tail": 500, "page": 64},
        # a serving step of a small batch: little is copied, latency counts
        {"name": "step-b12", "kind": "step", "model": "llama8b", "layers": 2, "slots": 12, "pages": 256, "page": 16,
         "tail": 200, "new": 1},
        # a pool half full of scattered pages, of every layer
        {"name": "compact-2k", "kind": "compact", "model": "llama8b", "layers": 32, "slots": 48, "pages": 2048,
         "page": 16, "tail": 500},
    ]


def draw(rng):
    """One more case: packed sequences of 1 to 9,000 tokens up to 40k rows, 1 to 20k rows of heads, contexts of 0 to
    124k rows with 1 to 96 sequences, pools of 64 to 4,096 pages of 8 to 64 rows."""
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["pack", "pack", "norm", "shared", "shared", "shared", "step", "compact"])
    model = rng.choice(sorted(MODELS))
    if kind == "pack":
        lens = rng.choice(["docs", "mixed", "even"])
        rows = log_int(40, 40000)
        seqs = min(rows, log_int(1, 300))
        if lens == "docs":
            seqs = max(1, rows // rng.randint(60, 400))
        return {"kind": kind, "model": model, "lens": lens, "seqs": max(seqs, -(-rows // 9000)), "rows": rows}
    if kind == "norm":
        return {"kind": kind, "model": model, "rows": log_int(1, 20000)}
    page = rng.choice([8, 16, 32, 64])
    if kind == "shared":
        new = rng.choice([1, 1, 1, rng.randint(2, 8)])
        slots = log_int(1, 96 // new)
        prefix = rng.choice([0] + [log_int(30, 124000)] * 7)
        return {"kind": kind, "model": model, "prefix": prefix, "slots": slots, "new": new,
                "tail": log_int(new, 800), "page": page}
    slots = log_int(4, 100)
    tail = log_int(20, 600)
    pages = max(64, slots * (3 + tail // page))
    layers = rng.choice([1, 4, 16, 32])
    return {"kind": kind, "model": model, "layers": layers, "slots": slots, "pages": pages, "page": page,
            "tail": tail, **({"new": rng.randint(1, 6)} if kind == "step" else {})}


# ---- shapes, the same for every seed ------------------------------------------
def _shape_rng(case):
    return random.Random("/".join("%s=%s" % (k, case[k]) for k in sorted(case) if k != "name"))


def _lens(case):
    """Sequence lengths of a packed batch, `rows` in all."""
    rng, n, rows = _shape_rng(case), case["seqs"], case["rows"]
    if case["lens"] == "even":
        return [rows // n + (i < rows % n) for i in range(n)]
    w = [rng.lognormvariate(0.0, 0.6 if case["lens"] == "docs" else 1.5) for _ in range(n)]
    lens = [max(1, int(x * (rows - n) / sum(w))) for x in w]
    if case["lens"] == "mixed" and n > 2:
        lens[n // 2] = 1
    most = 512 if case["lens"] == "docs" else 9000
    lens = [min(x, most) for x in lens]
    left = rows - sum(lens)
    for i in range(100 * n):  # what the limits cut goes to the shorter ones
        add = min(left, max(0, most - lens[i % n]), max(1, rows // n))
        lens[i % n] += add
        left -= add
    lens[0] += left
    return lens


def _tails(case):
    """Rows that each sequence has of its own, its new tokens among them; one slot in nine is idle."""
    rng = _shape_rng(case)
    return [0 if i % 9 == 5 else max(case["new"], int(case["tail"] * rng.uniform(0.3, 1.7)))
            for i in range(case["slots"])]


def _cdiv(a, b):
    return -(-a // b)


def _fitted(lens, page, room):
    """The lengths, halved until they fit `room` pages (or are a single page each)."""
    while sum(_cdiv(x, page) for x in lens) > room and max(lens) > page:
        lens = [_cdiv(x, 2) for x in lens]
    return lens


def _step_shape(case):
    """Of one serving step: lengths before it, rows kept, whose sequence a slot continues, new rows."""
    rng, n = _shape_rng(case), case["slots"]
    live = [i % 4 != 3 for i in range(n)]
    lens = [max(1, int(case["tail"] * rng.uniform(0.2, 1.6))) if x else 0 for x in live]
    lens = _fitted(lens, case["page"], case["pages"] - n * (1 + _cdiv(case["new"], case["page"])))
    keep = [-1] * n
    for i in range(0, n, 5):
        keep[i] = 0 if i % 2 else max(0, lens[i] - rng.randint(0, 3))
    heads = [i for i in range(n) if live[i] and keep[i] != 0 and i % 3 == 0] or [0]
    src = [rng.choice(heads) if not live[i] or keep[i] == 0 else -1 for i in range(n)]
    return lens, keep, src, [case["new"] if i % 7 != 6 else 0 for i in range(n)]


def _step_copies(case):
    """Pages copied before they are written: a shared, partly filled last page, but for its last holder."""
    lens, keep, src, new = _step_shape(case)
    after = [min(x, k) if k >= 0 else x for x, k in zip(lens, keep)]
    holder = [s if s >= 0 else i for i, s in enumerate(src)]
    held = [h for h in holder]
    after = [after[h] for h in holder]
    copies = 0
    for h in set(held):
        who = [i for i in range(len(held)) if held[i] == h]
        writes = sum(new[i] > 0 for i in who)
        if after[h] % case["page"] and len(who) > 1:
            copies += min(writes, len(who) - 1)
    return copies


def _compact_lens(case):
    rng = _shape_rng(case)
    lens = [max(1, int(case["tail"] * rng.uniform(0.2, 1.6))) for _ in range(case["slots"])]
    return _fitted(lens, case["page"], 0.6 * case["pages"])


def _max_pages(case):
    if case["kind"] == "shared":
        return max(1, max(_cdiv(x, case["page"]) for x in _tails(case)) + 1)
    return _cdiv(2 * case["tail"] + case.get("new", 0) + 1, case["page"]) + 1


# ---- inputs ---------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _bf16(g, *shape, scale=None):
    """Gaussian draws in slices (the float32 temporaries stay small), each channel with a scale of its own."""
    out = torch.empty(shape, dtype=BF, device=DEV)
    flat = out.view(-1, shape[-1])
    step = max(1, (1 << 27) // shape[-1])
    for i in range(0, flat.shape[0], step):
        x = torch.randn((min(step, flat.shape[0] - i), shape[-1]), generator=g, device=DEV)
        flat[i:i + step] = (x if scale is None else x * scale).to(BF)
    return out


def _channels(g):
    return torch.exp(0.5 * torch.randn(D, generator=g, device=DEV))


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _inv_freq():
    return THETA ** (-2.0 * torch.arange(D // 2, dtype=torch.float64, device=DEV) / D)


def _pool(g, layers, pages, page, hkv):
    """Keys and values of a pool: stale rows of earlier sequences wherever no sequence has written yet."""
    return _bf16(g, layers, pages, page, hkv, D), _bf16(g, layers, pages, page, hkv, D)


def _place(lens, pages, page, mp, g):
    """Tables of mp entries over randomly chosen pages, and the pages' reference counts."""
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    have = torch.tensor([_cdiv(x, page) for x in lens], device=DEV)
    first = torch.cumsum(have, 0) - have
    c = torch.arange(mp, device=DEV)
    at = (first[:, None] + c).clamp(max=pages - 1)
    used = c < have[:, None]
    table = torch.where(used, order[at], -1).to(torch.int32).contiguous()
    ref = torch.zeros(pages, dtype=torch.int32, device=DEV)
    ref[table[used].long()] = 1
    return table, ref, _i32(lens)


def prepare(case, seed):
    g = _gen(seed)
    hq, hkv = MODELS[case["model"]]
    kind = case["kind"]
    st = {"kind": kind, "hq": hq, "hkv": hkv}
    if own:
        import paper_2609_09768_amd as K
        st["K"] = K
    if kind == "pack":
        lens, n = _lens(case), case["rows"]
        st.update(n=n, q=_bf16(g, n, hq, D), k=_bf16(g, n, hkv, D, scale=_channels(g)), v=_bf16(g, n, hkv, D),
                  out=torch.empty((n, hq, D), dtype=BF, device=DEV), lse=torch.empty((n, hq), device=DEV))
        if own:
            st["pack"] = pack = K.Pack(lens, hq, hkv, D)
            pb = K.kvc_pack_plan_bytes(pack)
            st["plan"] = K.kvc_pack_plan_upload(pack, torch.empty(pb, dtype=torch.uint8, device=DEV), pb)
            st["wb"] = K.kvc_packed_attention_workspace(pack)
            st["ws"] = torch.empty(max(16, st["wb"]), dtype=torch.uint8, device=DEV)
        else:
            st["groups"] = _groups(lens, hq)
    elif kind == "norm":
        n, h = case["rows"], hq + 2 * hkv
        st.update(n=n, y=_bf16(g, n, h * D), gq=(1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(BF),
                  gk=(1 + 0.2 * torch.randn(D, generator=g, device=DEV)).to(BF),
                  pos=torch.sort(torch.randint(0, 124256, (n,), generator=g, device=DEV))[0].to(torch.int32),
                  q=torch.empty((n, hq, D), dtype=BF, device=DEV), k=torch.empty((n, hkv, D), dtype=BF, device=DEV),
                  v=torch.empty((n, hkv, D), dtype=BF, device=DEV), f=_inv_freq())
    elif kind == "shared":
        tails, mp = _tails(case), _max_pages(case)
        pages = max(1, sum(_cdiv(x, case["page"]) for x in tails)) + 3
        table, ref, length = _place(tails, pages, case["page"], mp, g)
        n, new, b = case["prefix"], case["new"], case["slots"]
        ch = _channels(g)
        st.update(n=n, new=new, table=table, len=length, page=case["page"], q=_bf16(g, b, new, hq, D),
                  kp=_bf16(g, n, hkv, D, scale=ch), vp=_bf16(g, n, hkv, D),
                  kt=_bf16(g, pages, case["page"], hkv, D, scale=ch), vt=_bf16(g, pages, case["page"], hkv, D),
                  out=torch.empty((b, new, hq, D), dtype=BF, device=DEV), lse=torch.empty((b, new, hq), device=DEV))
        if own:
            st["P"] = P = K.Pages(pages, case["page"], b, mp, ref, table, length)
            st["wb"] = K.kvc_shared_prefix_workspace(P, n, new, hq, hkv, D)
            st["ws"] = torch.empty(max(16, st["wb"]), dtype=torch.uint8, device=DEV)
    else:
        if kind == "step":
            lens, keep, src, new = _step_shape(case)
            st.update(keep=_i32(keep), src=_i32(src), new=_i32(new), max_new=case["new"])
        else:
            lens = _compact_lens(case)
        b, pages = case["slots"], case["pages"]
        table, ref, length = _place(lens, pages, case["page"], _max_pages(case), g)
        kp, vp = _pool(g, case["layers"], pages, case["page"], hkv)
        st.update(before=(ref, table, length), now=tuple(x.clone() for x in (ref, table, length)), kp=kp, vp=vp,
                  page=case["page"], layers=case["layers"])
        if own:
            st["P"] = P = K.Pages(pages, case["page"], b, table.shape[1], *st["now"])
            st["wb"] = K.kvc_pages_workspace(P)
            st["ws"] = torch.empty(max(16, st["wb"]), dtype=torch.uint8, device=DEV)
            st.update(rows=torch.empty((b, case.get("new", 1)), dtype=torch.int32, device=DEV),
                      a=torch.empty(max(b, pages // 2), dtype=torch.int32, device=DEV),
                      z=torch.empty(max(b, pages // 2), dtype=torch.int32, device=DEV),
                      two=torch.empty(2, dtype=torch.int32, device=DEV))
    return st


def _groups(lens, hq):
    """Of the plain form: sequences of similar length, padded to the longest of them, as many at a time as keep the
    scores below 1.5e9 values.  Rows of the batch, and each row's place in the padded group."""
    start = [0]
    for x in lens:
        start.append(start[-1] + x)
    order, groups = sorted((i for i in range(len(lens)) if lens[i]), key=lambda i: -lens[i]), []
    while order:
        L = lens[order[0]]
        most = max(1, int(1.5e9 // (hq * L * L)))
        part = [i for i in order[:most] if 2 * lens[i] >= L or L <= 128]
        order = order[len(part):]
        first = torch.tensor([start[i] for i in part], device=DEV)
        n = torch.tensor([lens[i] for i in part], device=DEV)
        at = torch.arange(L, device=DEV)
        inside = at < n[:, None]
        rows = torch.where(inside, first[:, None] + at, first[:, None])
        flat = torch.nonzero(inside.reshape(-1)).reshape(-1)
        groups.append((rows, inside, rows.reshape(-1)[flat], flat))
    return groups


# ---- one pass --------------------------------------------------------------------
def run(st):
    return {"pack": _pack, "norm": _norm, "shared": _shared, "step": _step, "compact": _compact}[st["kind"]](st)


def _pack(st):
    hq, hkv = st["hq"], st["hkv"]
    if own:
        st["K"].kvc_packed_attention(st["pack"], st["plan"], st["q"], st["k"], st["v"], st["n"], 0.0, st["out"],
                                     st["lse"], st["ws"], st["wb"])
        return st["out"], st["lse"]
    grp = hq // hkv
    for rows, inside, to, flat in st["groups"]:
        n, L = rows.shape
        q = st["q"][rows].float().view(n, L, hkv, grp, D).permute(0, 2, 3, 1, 4).reshape(n, hkv, grp * L, D)
        k = st["k"][rows].float().permute(0, 2, 3, 1).contiguous()
        v = st["v"][rows].float().permute(0, 2, 1, 3).contiguous()
        s = (q @ k).mul_(1.0 / math.sqrt(D)).view(n, hkv, grp, L, L)
        at = torch.arange(L, device=DEV)
        s.masked_fill_(at > at[:, None], -INF)
        top = s.amax(-1, keepdim=True)
        p = s.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        o = (p.view(n, hkv, grp * L, L) @ v).view(n, hkv, grp, L, D) / total
        st["out"][to] = o.permute(0, 3, 1, 2, 4).reshape(n * L, hq, D)[flat].to(BF)
        st["lse"][to] = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(n * L, hq)[flat]
    return st["out"], st["lse"]


def _norm(st):
    n, hq, hkv = st["n"], st["hq"], st["hkv"]
    if own:
        st["K"].kvc_qkv_norm_rope(st["y"], n, hq, hkv, hkv, D, st["gq"], st["gk"], EPS, st["pos"], THETA, st["q"],
                                  st["k"], st["v"])
        return st["q"], st["k"], st["v"]
    y = st["y"].view(n, hq + 2 * hkv, D)
    a = st["pos"].double()[:, None] * st["f"]
    cos, sin = a.cos().float()[:, None], a.sin().float()[:, None]

    def head(x, gamma):
        x = x.float()
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gamma.float()
        lo, hi = x[..., :D // 2], x[..., D // 2:]
        return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1).to(BF)

    return head(y[:, :hq], st["gq"]), head(y[:, hq:hq + hkv], st["gk"]), y[:, hq + hkv:].contiguous()


def _shared(st):
    hq, hkv, n, new = st["hq"], st["hkv"], st["n"], st["new"]
    if own:
        st["K"].kvc_shared_prefix_attention(st["q"], new, st["kp"], st["vp"], n, st["P"], st["kt"], st["vt"], hq, hkv,
                                            D, 0.0, st["out"], st["lse"], st["ws"], st["wb"])
        return st["out"], st["lse"]
    b, mp = st["table"].shape
    grp, m = hq // hkv, mp * st["page"]
    q = st["q"].float().mul(1.0 / math.sqrt(D)).view(b, new, hkv, grp, D).permute(2, 0, 1, 3, 4)
    kp, vp = st["kp"].float().permute(1, 2, 0).contiguous(), st["vp"].float().permute(1, 0, 2).contiguous()
    sp = (q.reshape(hkv, b * new * grp, D) @ kp).view(hkv, b, new, grp, n)
    at = st["table"].long().clamp(min=0)
    kt = st["kt"][at].view(b, m, hkv, D).float().permute(2, 0, 3, 1).contiguous()
    vt = st["vt"][at].view(b, m, hkv, D).float().permute(2, 0, 1, 3).contiguous()
    t = st["len"].long()[:, None] - new + torch.arange(new, device=DEV)
    seen = torch.arange(m, device=DEV) <= t[:, :, None]
    ss = (q.reshape(hkv, b, new * grp, D) @ kt).view(hkv, b, new, grp, m).masked_fill(~seen[:, :, None], -INF)
    top = torch.maximum(sp.amax(-1, keepdim=True) if n else torch.full_like(ss[..., :1], -INF),
                        ss.amax(-1, keepdim=True))
    live = (t >= 0)[None, :, :, None, None]
    top = torch.where(live, top, 0.0)
    ep, es = (sp - top).exp(), (ss - top).exp()
    total = ep.sum(-1, keepdim=True) + es.sum(-1, keepdim=True)
    o = (ep.view(hkv, b * new * grp, n) @ vp).view(hkv, b, new, grp, D) + \
        (es.view(hkv, b, new * grp, m) @ vt).view(hkv, b, new, grp, D)
    o = torch.where(live, o / total, 0.0).permute(1, 2, 0, 3, 4).reshape(b, new, hq, D)
    lse = torch.where(live, top + total.log(), -INF).permute(1, 2, 0, 3, 4).reshape(b, new, hq)
    return o.to(BF), lse


def _plain_copy(pool, src, dst):
    pool[:, dst] = pool[:, src]


def _entries(table, lens, page):
    return torch.arange(table.shape[1], device=DEV) < ((lens + page - 1) // page)[:, None]


def _counted(ref, table, mask, sign):
    """Reference counts with those of the marked table entries added or taken off."""
    return ref.index_add(0, table.long().clamp(min=0).reshape(-1), (sign * mask.reshape(-1)).to(torch.int32))


def _step(st):
    for x, y in zip(st["now"], st["before"]):
        x.copy_(y)
    page, max_new = st["page"], st["max_new"]
    if own:
        K, P, b = st["K"], st["P"], st["src"].shape[0]
        hkv, ws, wb, a, z = st["hkv"], st["ws"], st["wb"], st["a"], st["z"]
        K.kvc_pages_trim(P, st["keep"])
        K.kvc_pages_fork(P, st["src"], ws, wb)
        K.kvc_pages_reserve(P, st["new"], max_new, st["rows"], a, z, st["two"], ws, wb)
        K.kvc_pages_copy(P, a, z, b, None, st["layers"], hkv, D, st["kp"], st["vp"])
        return [*st["now"], st["rows"], a[:b], z[:b], st["two"], st["kp"], st["vp"]]
    ref, table, lens = st["now"]
    pages, (b, mp) = ref.shape[0], table.shape
    # rows that stay
    kept = torch.where((st["keep"] >= 0) & (st["keep"] < lens), st["keep"], lens)
    ref = _counted(ref, table, _entries(table, lens, page) & ~_entries(table, kept, page), -1)
    lens = kept
    # slots that go on with another's sequence
    fork = (st["src"] >= 0) & (st["src"] < b) & (st["src"] != torch.arange(b, device=DEV))
    src = torch.where(fork, st["src"], 0).long()
    ref = _counted(ref, table, _entries(table, lens, page) & fork[:, None], -1)
    theirs = _entries(table, lens, page)[src] & fork[:, None]
    table = torch.where(theirs, table[src], table)
    lens = torch.where(fork, lens[src], lens)
    ref = _counted(ref, table, theirs, 1)
    # rows for the new tokens
    new = st["new"].clamp(0, max_new)
    have, need = (lens + page - 1) // page, (lens + new + page - 1) // page
    last = table.gather(1, (have - 1).clamp(min=0).long()[:, None]).squeeze(1)
    part = (lens % page != 0) & (new > 0)
    same = (last[:, None] == last) & part[:, None] & part
    before = same.tril(-1).sum(1)
    fresh = part & (ref[last.long().clamp(min=0)] - before > 1)
    count = torch.where(new > 0, need - have, 0) + fresh
    first = torch.cumsum(count, 0) - count
    free = ref == 0
    missing = (count.sum() - free.sum()).clamp(min=0)
    full = (need > mp).sum()
    good = (missing == 0) & (full == 0)
    turn = torch.where(free, torch.cumsum(free, 0) - 1, pages)
    by_turn = torch.full((pages + 1,), -1, dtype=torch.int32, device=DEV).scatter(
        0, turn, torch.arange(pages, dtype=torch.int32, device=DEV))
    fresh, new = fresh & good, torch.where(good, new, 0)
    c = torch.arange(mp, device=DEV)
    added = (c >= have[:, None]) & (c < need[:, None]) & (new > 0)[:, None]
    moved = fresh[:, None] & (c == have[:, None] - 1)
    at = first[:, None] + torch.where(moved, 0, fresh[:, None] + c - have[:, None])
    put = torch.where(added | moved, by_turn[at.clamp(0, pages)], -1)
    copy_src, copy_dst = torch.where(fresh, last, -1), torch.where(moved, put, -1).amax(1)
    ref = _counted(ref, table, moved, -1)
    table = torch.where(added | moved, put, table)
    ref = _counted(ref, table, added | moved, 1)
    r = torch.arange(max_new, device=DEV)
    t = (lens[:, None] + r).clamp(max=mp * page - 1)
    rows = torch.where(r < new[:, None], table.gather(1, (t // page).long()) * page + t % page, -1).to(torch.int32)
    lens = lens + new
    on = copy_dst >= 0
    s, d = copy_src[on].long(), copy_dst[on].long()
    _plain_copy(st["kp"], s, d)
    _plain_copy(st["vp"], s, d)
    for x, y in zip(st["now"], (ref, table, lens)):
        x.copy_(y)
    return [*st["now"], rows, copy_src.to(torch.int32), copy_dst.to(torch.int32),
            torch.stack([missing, full]).to(torch.int32), st["kp"], st["vp"]]


def _compact(st):
    for x, y in zip(st["now"], st["before"]):
        x.copy_(y)
    ref, table, lens = st["now"]
    pages, half = ref.shape[0], ref.shape[0] // 2
    if own:
        K, P, hkv, ws, wb = st["K"], st["P"], st["hkv"], st["ws"], st["wb"]
        K.kvc_pages_compact(P, st["a"], st["z"], st["two"], ws, wb)
        K.kvc_pages_copy(P, st["a"], st["z"], half, st["two"][1:], st["layers"], hkv, D, st["kp"], st["vp"])
        return [*st["now"], st["a"][:half], st["z"][:half], st["two"], st["kp"], st["vp"]]
    live = ref > 0
    count = live.sum()
    number = torch.arange(pages, device=DEV)
    far, hole = live & (number >= count), ~live & (number < count)
    s, d = torch.nonzero(far).squeeze(1), torch.nonzero(hole).squeeze(1)
    to = number.scatter(0, s, d)
    used = _entries(table, lens, st["page"])
    table.copy_(torch.where(used, to[table.long().clamp(min=0)].to(torch.int32), table))
    ref[d] = ref[s]
    ref[s] = 0
    move = torch.full((2, half), -1, dtype=torch.int32, device=DEV)
    move[0, :s.shape[0]], move[1, :s.shape[0]] = s.to(torch.int32), d.to(torch.int32)
    _plain_copy(st["kp"], s, d)
    _plain_copy(st["vp"], s, d)
    return [ref, table, lens, move[0], move[1], torch.stack([count, far.sum()]).to(torch.int32), st["kp"], st["vp"]]


# ---- what a pass cannot do without -------------------------------------------------
def work(case):
    hq, hkv = MODELS[case["model"]]
    kind = case["kind"]
    if kind == "pack":
        return {"bytes": case["rows"] * ((2 * hq + 2 * hkv) * D * 2 + hq * 4),
                "flops": 4 * D * hq * sum(x * (x + 1) // 2 for x in _lens(case))}
    if kind == "norm":
        n, h = case["rows"], hq + 2 * hkv
        return {"bytes": n * (h * D * 4 + 4) + 4 * D, "flops": n * (hq + hkv) * D * 7}
    if kind == "shared":
        tails, n, new = _tails(case), case["prefix"], case["new"]
        return {"bytes": (n + sum(tails)) * hkv * D * 4 + len(tails) * new * hq * (4 * D + 4),
                "flops": 4 * D * hq * new * (sum(x > 0 for x in tails) * n + sum(tails))}
    one = case["layers"] * 2 * case["page"] * hkv * D * 2  # a page of every layer, keys and values
    if kind == "step":
        return {"bytes": 2 * one * _step_copies(case) + 8 * case["pages"] + 16 * case["slots"], "flops": 0}
    used = sum(_cdiv(x, case["page"]) for x in _compact_lens(case))
    moves = used * (case["pages"] - used) / case["pages"]
    return {"bytes": 2 * one * moves + 8 * case["pages"] + 8 * used, "flops": 0}


# ---- the same in 64 bits, from the definitions ---------------------------------------
def _soft(q, k, v, sees):
    """Rows of q [r, D] over keys [n, D], row i the first sees[i] of them: attention and log-sum, in float64."""
    s = (q @ k.T) / math.sqrt(D)
    s[torch.arange(k.shape[0], device=DEV) >= sees[:, None]] = -INF
    m = s.max(1)[0].clamp(min=-1e300)
    e = torch.exp(s - m[:, None])
    z = e.sum(1)
    return (e @ v) / z.clamp(min=1e-300)[:, None], m + torch.log(z)


def exact(case, seed):
    global own
    if case["kind"] in ("step", "compact"):
        return None
    was, own = own, False
    st = prepare(case, seed)
    own = was
    hq, hkv = st["hq"], st["hkv"]
    grp = hq // hkv
    if case["kind"] == "norm":
        n, h = st["n"], hq + hkv
        y = st["y"].view(n, h + hkv, D).double()
        f = torch.tensor([math.pow(THETA, -2.0 * j / D) for j in range(D // 2)], dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV), st["pos"].double()[:, None] * f)[:, None]
        gamma = torch.cat([st["gq"].double().expand(hq, D), st["gk"].double().expand(hkv, D)])
        x = y[:, :h] * gamma * torch.rsqrt(y[:, :h].pow(2).sum(-1, keepdim=True) / D + EPS)
        z = torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) * turn
        x = torch.cat([z.real, z.imag], -1)
        return x[:, :hq].contiguous(), x[:, hq:].contiguous(), None
    out, lse = st["out"].double().zero_(), st["lse"].double().zero_()
    if case["kind"] == "pack":
        lo = 0
        for L in _lens(case):
            for h in range(hq):
                for i in range(lo, lo + L, 4096):
                    j = min(i + 4096, lo + L)
                    out[i:j, h], lse[i:j, h] = _soft(
                        st["q"][i:j, h].double(), st["k"][lo:j, h // grp].double(), st["v"][lo:j, h // grp].double(),
                        torch.arange(i - lo + 1, j - lo + 1, device=DEV))
            lo += L
        return out, lse
    n, new, page = st["n"], st["new"], st["page"]
    lse.fill_(-INF)
    for b, own_rows in enumerate(_tails(case)):
        if not own_rows:
            continue
        at = torch.arange(own_rows, device=DEV)
        pg = st["table"][b].long()[at // page]
        k, v = (torch.cat([x, y[pg, at % page]]) for x, y in ((st["kp"], st["kt"]), (st["vp"], st["vt"])))
        t = own_rows - new + torch.arange(new, device=DEV)
        sees = torch.where(t >= 0, n + t + 1, 0).repeat_interleave(grp)
        for g in range(hkv):
            o, z = _soft(st["q"][b, :, g * grp:(g + 1) * grp].reshape(new * grp, D).double(), k[:, g].double(),
                         v[:, g].double(), sees)
            out[b, :, g * grp:(g + 1) * grp] = o.view(new, grp, D)
            lse[b, :, g * grp:(g + 1) * grp] = z.view(new, grp)
    return out, lse
