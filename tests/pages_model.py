"""The pages of a cache in plain Python: the definition that the library's calls are
compared with (include/grkv.h), one entry, page and row at a time."""
import numpy as np

OK, FULL, LENGTH, UNIT, RANGE = 0, 1, 2, 3, 4


class PagesModel:
    """Rows are Python objects (or arrays); k and v of a slot travel together."""

    def __init__(self, units, max_pages, pages, page_size):
        self.units, self.max_pages, self.ps = units, max_pages, page_size
        self.refs = [0] * pages
        self.table = [[] for _ in range(units)]
        self.lens = [0] * units
        self.data = {}   # (page, row) -> (k, v)

    # --- what a call sees before it writes anything

    def _ceil(self, n):
        return -(-n // self.ps)

    def _owners(self, dst):
        own = {}
        for i, w in enumerate(dst):
            if 0 <= w < self.units:
                own.setdefault(w, i)
        return own

    def slot(self, u, s):
        return self.data.get((self.table[u][s // self.ps], s % self.ps))

    def _run(self, plans):
        """plans: (status, dst, pages kept, new pages, length, rows of the new slots) per entry,
        in order; hands out pages in order, then gives up the old ones."""
        status, done, short = [], [], False
        low = 0
        for st, src, dst, keep, need, n1, rows, first_slot in plans:
            if st == OK and need > 0:
                free = [p for p, r in enumerate(self.refs) if r == 0][:need] if not short else []
                if short or len(free) < need:
                    st, short = FULL, True
                else:
                    for p in free:
                        self.refs[p] = 1
            else:
                free = []
            status.append(st)
            if st in (OK, RANGE) and n1 is not None:
                done.append((src, dst, keep, free, n1, rows, first_slot))
        for src, dst, keep, free, n1, rows, first_slot in done:
            if src != dst:
                for p in keep:
                    self.refs[p] += 1
            else:
                for p in self.table[dst][len(keep):]:
                    self.refs[p] -= 1
            self.table[dst], self.lens[dst] = keep + free, n1
            for i, r in enumerate(rows):
                s = first_slot + i
                self.data[(self.table[dst][s // self.ps], s % self.ps)] = r
        return status

    def append(self, units, rows, bad=()):
        """rows[i]: the (k, v) rows of entry i; bad: entries whose source is out of range."""
        own, plans = self._owners(units), []
        for i, (u, r) in enumerate(zip(units, rows)):
            if not 0 <= u < self.units or own[u] != i:
                plans.append((UNIT, u, u, [], 0, None, [], 0))
                continue
            n0 = self.lens[u]
            n1 = n0 + len(r)
            st = RANGE if i in bad else LENGTH if n1 > self.max_pages * self.ps else OK
            plans.append((st, u, u, list(self.table[u]), self._ceil(n1) - self._ceil(n0),
                          n1 if st == OK else None, r, n0))
        return self._run(plans)

    def compact(self, src, dst, keep, idx, bad=()):
        """idx[i]: the slots of entry i behind its first keep[i] (None: fork, keep all)."""
        own, plans = self._owners(dst), []
        zero = None
        wrong = set()
        for i, (u, w) in enumerate(zip(src, dst)):
            refused = (not 0 <= u < self.units or not 0 <= w < self.units or own.get(w) != i
                       or (u != w and (u in own or self.lens[w] != 0)))
            if refused:
                plans.append((UNIT, u, w, [], 0, None, [], 0))
                continue
            n0 = self.lens[u]
            kp = n0 if keep is None else keep[i]
            pick = [] if keep is None else list(idx[i])
            n1 = kp + len(pick)
            st = OK
            if not 0 <= kp <= n0 or i in bad:
                st = RANGE
            elif n1 > self.max_pages * self.ps:
                st = LENGTH
            if st != OK:
                plans.append((st, u, w, [], 0, None, [], 0))
                continue
            first = kp // self.ps
            if u == w and not pick and kp % self.ps and self.refs[self.table[u][first]] == 1:
                first += 1
            rows = []
            for s in range(first * self.ps, n1):
                f = s if s < kp else pick[s - kp]
                if 0 <= f < n0:
                    rows.append(self.slot(u, f))
                else:
                    rows.append(zero)
                    wrong.add(i)
            plans.append((OK, u, w, self.table[u][:first], max(0, self._ceil(n1) - first), n1,
                          rows, first * self.ps))
        status = self._run(plans)
        return [RANGE if s == OK and i in wrong else s for i, s in enumerate(status)]

    def fork(self, src, dst):
        return self.compact(src, dst, None, None)

    def free(self, units):
        status = []
        for u in units:
            ok = 0 <= u < self.units
            status.append(OK if ok else UNIT)
            if ok:
                for p in self.table[u]:
                    self.refs[p] -= 1
                self.table[u], self.lens[u] = [], 0
        return status

    # --- state as arrays

    def arrays(self):
        table = np.full((self.units, self.max_pages), -1, np.int32)
        for u, r in enumerate(self.table):
            table[u, :len(r)] = r
        words = np.zeros(-(-len(self.refs) // 32), np.uint32)
        for p, r in enumerate(self.refs):
            if r == 0:
                words[p // 32] |= np.uint32(1 << (p % 32))
        return table, np.array(self.lens, np.int32), np.array(self.refs, np.int32), words.view(np.int32)
