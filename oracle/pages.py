"""Pages of a cache pool, one step after the other (test infrastructure only).

Slot s holds len[s] rows; row r is row r % page_rows of page
table[s][r // page_rows]; ref[p] counts the table entries that hold page p.
The steps are written the way a serving loop would do them by hand, slot by
slot, taking the lowest free page each time.
"""
import numpy as np


class PageTables:
    def __init__(self, n_pages, page_rows, n_slots, max_pages):
        self.page_rows, self.max_pages = page_rows, max_pages
        self.ref = np.zeros(n_pages, dtype=np.int32)
        self.table = np.full((n_slots, max_pages), -1, dtype=np.int32)
        self.len = np.zeros(n_slots, dtype=np.int32)

    def copy(self):
        t = PageTables(len(self.ref), self.page_rows, len(self.len), self.max_pages)
        t.ref, t.table, t.len = self.ref.copy(), self.table.copy(), self.len.copy()
        return t

    def held(self, s):
        """Pages of slot s, in order."""
        n = -(-int(self.len[s]) // self.page_rows)
        return [int(p) for p in self.table[s, :n]]

    def trim(self, keep):
        for s, k in enumerate(keep):
            if 0 <= k < self.len[s]:
                for p in self.held(s)[-(-int(k) // self.page_rows):]:
                    self.ref[p] -= 1
                self.len[s] = k

    def fork(self, src_of):
        old = self.copy()
        for s, a in enumerate(src_of):
            if 0 <= a < len(self.len) and a != s:
                for p in old.held(s):
                    self.ref[p] -= 1
                for c, p in enumerate(old.held(a)):
                    self.table[s, c] = p
                    self.ref[p] += 1
                self.len[s] = old.len[a]

    def reserve(self, n_new, max_new):
        """rows, copy_src, copy_dst, shortage; nothing changes if a page or a table entry is missing."""
        t, n = self.copy(), len(self.len)
        rows = np.full((n, max_new), -1, dtype=np.int32)
        src, dst = np.full(n, -1, dtype=np.int32), np.full(n, -1, dtype=np.int32)
        free = [int(p) for p in np.nonzero(t.ref == 0)[0]]
        missing = full = 0

        def take():
            nonlocal missing
            if free:
                return free.pop(0)
            missing += 1
            return -1

        for s in range(n):
            w = min(max(int(n_new[s]), 0), max_new)
            if w == 0:
                continue
            have, pr = int(t.len[s]), self.page_rows
            held, need = -(-have // pr), -(-(have + w) // pr)
            full += need > self.max_pages
            if have % pr and t.ref[t.table[s, held - 1]] > 1:
                src[s], dst[s] = t.table[s, held - 1], take()
                t.ref[src[s]] -= 1
                if dst[s] >= 0:
                    t.ref[dst[s]] = 1
                t.table[s, held - 1] = dst[s]
            for c in range(held, need):
                p = take()
                if p >= 0:
                    t.ref[p] = 1
                if c < self.max_pages:
                    t.table[s, c] = p
            if not missing and not full:
                for i in range(w):
                    rows[s, i] = t.table[s, (have + i) // pr] * pr + (have + i) % pr
            t.len[s] = have + w
        if missing or full:
            rows[:], src[:], dst[:] = -1, -1, -1
        else:
            self.ref, self.table, self.len = t.ref, t.table, t.len
        return rows, src, dst, np.array([missing, full], dtype=np.int32)

    def compact(self):
        """move_src, move_dst, counts."""
        live = int((self.ref > 0).sum())
        far = [p for p in range(live, len(self.ref)) if self.ref[p] > 0]
        holes = [p for p in range(live) if self.ref[p] == 0]
        move = np.full((2, len(self.ref) // 2), -1, dtype=np.int32)
        to = dict(zip(far, holes))
        for i, (a, b) in enumerate(to.items()):
            move[:, i] = a, b
            self.ref[b], self.ref[a] = self.ref[a], 0
        for s in range(len(self.len)):
            for c, p in enumerate(self.held(s)):
                self.table[s, c] = to.get(p, p)
        return move[0], move[1], np.array([live, len(far)], dtype=np.int32)
