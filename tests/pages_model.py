"""The page operators as a program that cares for one page after another on the host would write them (numpy)."""
import numpy as np

DONE, NONE_LEFT, REFUSED = 0, 1, 2


class Model:
    def __init__(self, k, v, table, lens, ref, ps):
        """k, v: [layers, pages, ...] arrays of any type; the rest int32."""
        self.k, self.v, self.table, self.lens, self.ref = (a.copy() for a in (k, v, table, lens, ref))
        self.ps = ps

    def _pages(self, n):
        return -(-int(n) // self.ps)

    def _copy(self, pairs):
        for src, dst in pairs:
            for cache in (self.k, self.v):
                cache[:, dst] = cache[:, src]

    def copy(self, src, dst):
        n = len(self.ref)
        self._copy([(s, d) for s, d in zip(src, dst) if 0 <= s < n and 0 <= d < n])

    def _serve(self, needs):
        """The free pages each request gets, None: the free ones do not reach."""
        free, at, out = [p for p in range(len(self.ref)) if self.ref[p] == 0], 0, []
        for need in needs:
            at += need
            out.append(free[at - need:at] if need == 0 or at <= len(free) else None)
        return out

    def _row_ok(self, r):
        return 0 <= r < len(self.lens) and 0 <= self.lens[r] <= self.table.shape[1] * self.ps

    def fork(self, parents, children):
        ok, seen = [], set()
        for p, c in zip(parents, children):
            good = self._row_ok(c) and self._row_ok(p) and p != c and self.lens[c] == 0 and c not in seen
            seen.add(c)
            ok.append(good)
        lens = self.lens.copy()
        got = self._serve([int(g and lens[p] % self.ps != 0) for g, p in zip(ok, parents)])
        status, copies, more, rows = [], [], [], []
        for g, fresh, p, c in zip(ok, got, parents, children):
            status.append(REFUSED if not g else NONE_LEFT if fresh is None else DONE)
            if status[-1] != DONE:
                continue
            pages = self.table[p, :self._pages(lens[p])].copy()
            if fresh:
                copies.append((pages[-1], fresh[0]))
                pages[-1] = fresh[0]
            rows.append((c, pages, lens[p]))
        for c, pages, n in rows:
            self.table[c, :len(pages)] = pages
            self.lens[c] = n
            np.add.at(self.ref, pages, 1)
        self._copy(copies)
        return status

    def resize(self, rows, lengths):
        ok, seen, needs, split = [], set(), [], []
        for r, n in zip(rows, lengths):
            good = self._row_ok(r) and 0 <= n <= self.table.shape[1] * self.ps and r not in seen
            seen.add(r)
            ok.append(good)
            need, part = 0, None
            if good:
                need = max(0, self._pages(n) - self._pages(self.lens[r]))
                if n < self.lens[r] and n % self.ps and self.ref[self.table[r, self._pages(n) - 1]] > 1:
                    need, part = 1, self.table[r, self._pages(n) - 1]
            needs.append(need)
            split.append(part)
        got, status, copies = self._serve(needs), [], []
        for g, fresh, part, r, n in zip(ok, got, split, rows, lengths):
            status.append(REFUSED if not g else NONE_LEFT if fresh is None else DONE)
            if status[-1] != DONE:
                continue
            had, has = self._pages(self.lens[r]), self._pages(n)
            np.subtract.at(self.ref, self.table[r, has:had], 1)
            if part is not None:
                self.ref[part] -= 1
                self.table[r, has - 1] = fresh[0]
                copies.append((part, fresh[0]))
            else:
                self.table[r, had:max(has, had)] = fresh
            self.ref[fresh] = 1
            self.lens[r] = n
        self._copy(copies)
        return status

    def compact(self):
        n, live = len(self.ref), [p for p in range(len(self.ref)) if self.ref[p] > 0]
        new_page = np.full(n, -1, dtype=np.int32)
        new_page[live] = live
        holes = [p for p in range(len(live)) if self.ref[p] == 0]
        moves = list(zip([p for p in live if p >= len(live)], holes))
        for src, dst in moves:
            new_page[src] = dst
            self.ref[dst], self.ref[src] = self.ref[src], 0
        for r in range(len(self.lens)):
            used = self.table[r, :self._pages(self.lens[r])]
            used[:] = new_page[used]
        self._copy(moves)
        return new_page, len(live)

    def counts(self):
        """References that the rows hold."""
        ref = np.zeros_like(self.ref)
        for r, n in enumerate(self.lens):
            np.add.at(ref, self.table[r, :self._pages(n)], 1)
        return ref
