"""Plain form, on lists and CPU tensors, of the calls that change a cache's pages (no code of the library)."""
from __future__ import annotations

import torch


def copy_of(cache, lens):
    """The cache and lengths on the CPU: {name: tensor}."""
    got = {n: getattr(cache, n) for n in ("k", "v", "k_scale", "v_scale", "table", "refs")}
    got["lens"] = lens
    return {n: None if x is None else (x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x).cpu().clone()
            for n, x in got.items()}


class Book:
    """A call's outcome from the state before it: sequences in order, entries in order, lowest free page first."""

    def __init__(self, state):
        self.s = state
        self.n_pages, self.Hkv, self.page, _ = state["k"].shape
        self.B, self.most = state["table"].shape
        self.old = state["table"].tolist()
        self.old_lens = None if state["lens"] is None else state["lens"].tolist()
        self.left = [p for p, n in enumerate(state["refs"].tolist()) if n == 0]
        self.stopped = False

    def named(self, p):
        return 0 <= p < self.n_pages

    def pages(self, rows):
        return -(-min(max(rows, 0), self.most * self.page) // self.page)

    def take(self, number):
        self.stopped = self.stopped or number > len(self.left)
        if number and self.stopped:
            return None
        got, self.left = self.left[:number], self.left[number:]
        return got

    def put(self, b, row, lens=None):
        for p in self.old[b]:
            if self.named(p):
                self.s["refs"][p] -= 1
        for p in row:
            if self.named(p):
                self.s["refs"][p] += 1
        self.s["table"][b] = torch.tensor(row, dtype=torch.int32)
        if lens is not None:
            self.s["lens"][b] = torch.tensor(lens, dtype=torch.int32)

    def hold(self, rows):
        missing = []
        for b, row in enumerate(rows.tolist()):
            new, need = list(self.old[b]), self.pages(max(row))
            gaps = [j for j in range(need) if not self.named(new[j])]
            got = self.take(len(gaps))
            missing.append(len(gaps) if got is None else 0)
            for j, p in zip(gaps, got or [-1] * len(gaps)):
                new[j] = p
            self.put(b, new[:need] + [-1] * (self.most - need))
        return missing

    def copy(self, frm, to):
        """Row (page, head, slot) `to` becomes row `frm` (None: zeros with scale 1) as it was."""
        for n in ("k", "v"):
            self.s[n][to] = 0 if frm is None else self.before[n][frm]
            if self.s[n + "_scale"] is not None:
                self.s[n + "_scale"][to] = 1.0 if frm is None else self.before[n + "_scale"][frm]

    def fork(self, src):
        self.before = {n: None if self.s[n] is None else self.s[n].clone() for n in ("k", "v", "k_scale", "v_scale")}
        missing = []
        for b, a in enumerate(src.tolist()):
            missing.append(0)
            if a == b or not 0 <= a < self.B:
                continue
            lens = [min(max(n, 0), self.most * self.page) for n in self.old_lens[a]]
            whole, used = min(lens) // self.page, self.pages(max(lens))
            want = [j for j in range(whole, used) if self.named(self.old[a][j])]
            got = self.take(len(want))
            if got is None:
                missing[b] = len(want)
                continue
            new = [p if j < whole and self.named(p) else -1 for j, p in enumerate(self.old[a])]
            for j, p in zip(want, got):
                new[j] = p
                for c, n in enumerate(lens):
                    for x in range(max(0, min(self.page, n - j * self.page))):
                        self.copy((self.old[a][j], c, x), (p, c, x))
            self.put(b, new, self.old_lens[a])
        return missing

    def compact(self, idx, counts):
        self.before = {n: None if self.s[n] is None else self.s[n].clone() for n in ("k", "v", "k_scale", "v_scale")}
        missing, n, cap = [], idx.shape[2], self.most * self.page
        for b, row in enumerate(counts.tolist()):
            missing.append(0)
            if max(row) < 0:
                continue
            keep = [min(max(x, 0), n) for x in row]
            got = self.take(self.pages(max(keep)))
            if got is None:
                missing[b] = self.pages(max(keep))
                continue
            for c, m in enumerate(keep):
                for i, t in enumerate(idx[b, c, :min(m, cap)].tolist()):
                    known = 0 <= t < min(self.old_lens[b][c], cap) and self.named(self.old[b][t // self.page])
                    self.copy((self.old[b][t // self.page], c, t % self.page) if known else None,
                              (got[i // self.page], c, i % self.page))
            self.put(b, got + [-1] * (self.most - len(got)), keep)
        return missing
