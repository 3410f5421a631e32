"""The pool of pages in plain Python: who holds which page, and what every sequence holds."""
import torch

import paper_2607_22586_gb300 as M
from tests import cache_ref as R


class Pool:
    """Tensors of a pool whose pages are all free, and the plain form beside them: `held[l][b][h]` lists a
    sequence's rows, (K, V) of one row each, in float64, None where nothing is known."""

    def __init__(self, L, B, H, d, kind, page, n_pages, max_pages):
        self.L, self.B, self.H, self.d, self.kind, self.page = L, B, H, d, kind, page
        self.n_pages, self.max_pages = n_pages, max_pages
        dev = "cuda"
        self.table = torch.full((L, B, H, max_pages), -1, dtype=torch.int32, device=dev)
        self.lens = torch.zeros((L, B, H), dtype=torch.int32, device=dev)
        self.refs = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        shape = (n_pages, page, d)
        if kind == "i8":
            self.kp, self.vp = (torch.randint(-127, 128, shape, dtype=torch.int8, device=dev) for _ in range(2))
            self.ks, self.vs = (torch.full(shape[:2], float("nan"), device=dev) for _ in range(2))
        else:
            self.kp, self.vp = (torch.full(shape, float("nan"), dtype=R.DT[kind], device=dev) for _ in range(2))
            self.ks = self.vs = None
        self.m_table = [[[[-1] * max_pages for _ in range(H)] for _ in range(B)] for _ in range(L)]
        self.m_refs = [0] * n_pages
        self.held = [[[[] for _ in range(H)] for _ in range(B)] for _ in range(L)]
        self.exhausted = False

    def struct(self):
        return M.make_cache(self.kp, self.vp, self.table, self.lens, self.ks, self.vs)

    def units(self):
        return [(l, b, h) for l in range(self.L) for b in range(self.B) for h in range(self.H)]

    def get(self, l, b, h, pos):
        pos = torch.as_tensor(pos, device="cuda").long()
        s = self.table[l, b, h].long()[pos // self.page] * self.page + pos % self.page
        out = []
        for pages, scales in ((self.kp, self.ks), (self.vp, self.vs)):
            x = pages.view(-1, self.d)[s].double()
            out.append(x * scales.view(-1)[s].double()[:, None] if self.kind == "i8" else x)
        return out

    # ---- the plain form ----
    def _take(self, wanted):
        """wanted: (l, b, h, entry, rows of the old page that stay)."""
        free = [p for p in range(self.n_pages) if self.m_refs[p] == 0]
        old = []
        for k, (l, b, h, i) in enumerate(wanted):
            row = self.m_table[l][b][h]
            old.append(row[i])
            row[i] = free[k] if k < len(free) else -1
            if row[i] >= 0:
                self.m_refs[row[i]] = 1
            else:
                self.exhausted = True
        for p in old:
            if p >= 0:
                self.m_refs[p] -= 1

    def _needed(self, l, b, h, start, stop):
        if start >= stop:
            return []
        row = self.m_table[l][b][h]
        return [(l, b, h, i) for i in range(start // self.page, (stop - 1) // self.page + 1)
                if row[i] < 0 or self.m_refs[row[i]] > 1]

    def reserve(self, new, lens):
        """lens: after the new rows were counted."""
        cap = self.page * self.max_pages
        wanted = []
        for l, b, h in self.units():
            n, end = new[b], int(lens[l][b][h])
            end = cap if end > 1 << 30 else max(end, 0)
            if n:
                wanted += self._needed(l, b, h, max(end - n, 0), min(end, cap))
        self._take(wanted)

    def release(self, which):
        for l, b, h in self.units():
            if b in which:
                for i, p in enumerate(self.m_table[l][b][h]):
                    if p >= 0:
                        self.m_refs[p] -= 1
                    self.m_table[l][b][h][i] = -1
                self.held[l][b][h] = []

    def fork(self, src, dst):
        self.release(dst)
        for s, t in zip(src, dst):
            for l in range(self.L):
                for h in range(self.H):
                    n = len(self.held[l][s][h])
                    pages = (n + self.page - 1) // self.page
                    for i in range(pages):
                        p = self.m_table[l][t][h][i] = self.m_table[l][s][h][i]
                        if p >= 0:
                            self.m_refs[p] += 1
                    self.held[l][t][h] = list(self.held[l][s][h])

    def compact(self, idx, rows, counts=None):
        """idx[l][cu_b + i][h]."""
        cu = R.cu_of(rows)
        wanted = []
        kept = {}
        for l, b, h in self.units():
            if rows[b]:
                m = min(rows[b], len(self.held[l][b][h]))
                if counts is not None:
                    m = min(m, max(int(counts[l][b][h]), 0))
                kept[l, b, h] = m
                wanted += self._needed(l, b, h, 0, m)
        self._take(wanted)
        for (l, b, h), m in kept.items():
            held = self.held[l][b][h]
            zero = torch.zeros(self.d, dtype=torch.float64, device="cuda")
            new = []
            for i in range(m):
                p = int(idx[l][cu[b] + i][h])
                new.append(held[p] if i <= p < len(held) else (zero, zero))
            self.held[l][b][h] = new
            for i in range((m + self.page - 1) // self.page, self.max_pages):
                p = self.m_table[l][b][h][i]
                if p >= 0:
                    self.m_refs[p] -= 1
                self.m_table[l][b][h][i] = -1

    def append(self, l, b, h, k, v):
        """Rows of the call, as the pages hold them."""
        if self.kind == "i8":
            k, v = ((c.double() * s.double()[:, None]) for c, s in (R.quantise(k), R.quantise(v)))
        self.held[l][b][h] += list(zip(k.double(), v.double()))

    def check(self, what=""):
        assert self.table.tolist() == self.m_table, (what, "table")
        assert self.refs.tolist() == self.m_refs, (what, "refs")
        assert self.lens.tolist() == [[[len(x) for x in y] for y in z] for z in self.held], (what, "lens")
        for l, b, h in self.units():
            held = self.held[l][b][h]
            pages = (len(held) + self.page - 1) // self.page
            # rows without a page are lost
            at = [i for i in range(len(held)) if self.m_table[l][b][h][i // self.page] >= 0]
            if not at:
                continue
            k, v = self.get(l, b, h, at)
            for x, j in ((k, 0), (v, 1)):
                want = torch.stack([held[i][j] for i in at])
                assert torch.equal(x, want), (what, l, b, h, "rows", pages)
