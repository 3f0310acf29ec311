"""The page-table oracle: counts follow the tables, rows never collide."""
import numpy as np
import pytest

import oracle


def _consistent(t):
    ref = np.zeros_like(t.ref)
    for s in range(len(t.len)):
        for p in t.held(s):
            ref[p] += 1
    return np.array_equal(ref, t.ref)


@pytest.mark.parametrize("seed", range(6))
def test_counts_follow_tables_and_contents_follow_sequences(seed):
    # every sequence's tokens, written through the rows, read back through the tables after each step
    rng = np.random.default_rng(seed)
    pr, slots, mp = int(rng.choice([8, 16])), 7, 6
    t = oracle.PageTables(int(rng.integers(12, 60)), pr, slots, mp)
    pool, seqs, token = np.zeros(len(t.ref) * pr, dtype=np.int64), [[] for _ in range(slots)], 0
    for _ in range(60):
        before = t.copy()
        want = np.minimum(rng.integers(0, 12, slots), mp * pr - t.len)
        rows, src, dst, short = t.reserve(want, 12)
        if short.any():
            assert (rows < 0).all() and (src < 0).all() and np.array_equal(before.table, t.table)
        for a, b in zip(src, dst):
            if a >= 0:
                pool[b * pr:(b + 1) * pr] = pool[a * pr:(a + 1) * pr]
        for s in range(slots):
            for r in rows[s][rows[s] >= 0]:
                pool[r] = token
                seqs[s].append(token)
                token += 1
        keep = np.where(rng.random(slots) < 0.4, rng.integers(0, mp * pr, slots), -1)
        t.trim(keep)
        seqs = [x[:k] if k >= 0 else x for x, k in zip(seqs, keep)]
        fork = np.where(rng.random(slots) < 0.4, rng.integers(0, slots, slots), -1)
        t.fork(fork)
        seqs = [list(seqs[a]) if a >= 0 else x for x, a in zip(seqs, fork)]
        if rng.random() < 0.3:
            a, b, counts = t.compact()
            moved = pool.copy()
            for x, y in zip(a[:counts[1]], b[:counts[1]]):
                moved[y * pr:(y + 1) * pr] = pool[x * pr:(x + 1) * pr]
            pool = moved
            assert (t.ref[:counts[0]] > 0).all() and not t.ref[counts[0]:].any()
        assert _consistent(t)
        for s in range(slots):
            got = [pool[t.table[s, r // pr] * pr + r % pr] for r in range(t.len[s])]
            assert got == seqs[s], s


def test_last_holder_keeps_the_page():
    t = oracle.PageTables(10, 8, 3, 2)
    t.reserve([5, 0, 0], 8)
    t.fork([-1, 0, 0])
    _, src, dst, _ = t.reserve([1, 1, 1], 1)
    assert src.tolist() == [0, 0, -1] and dst.tolist() == [1, 2, -1] and t.ref[:3].tolist() == [1, 1, 1]
