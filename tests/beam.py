"""Beam search's selection and pool of pages by plain loops (not a test module): what the GPU tests compare with."""
import math

import torch

F32 = 2.0 ** -24                                  # half a step, relative to the value


def select(logits, n_groups, n_beams, score, n_out, scale=None, last=None, eos=-1, alpha=0.0, length=None):
    """(parent, token, score, length, bad rows) in 64 bits, candidate by candidate.  length: of each row, or None."""
    parent, token, value, new_len, bad = [], [], [], [], set()
    for g in range(n_groups):
        found = []
        for b in range(n_beams):
            r = g * n_beams + b
            s, c, n = float(score[r]), 1.0 if scale is None else float(scale[r]), 0 if length is None else int(length[r])
            if math.isnan(s) or s == math.inf or not 0 <= n < 2**31 - 1:
                bad.add(r)
                continue
            if s == -math.inf:
                continue
            if last is not None and eos >= 0 and int(last[r]) == eos:
                found.append((-s / max(n, 1) ** alpha, b, 0, eos, s, n))
                continue
            if not 0.0 < c < math.inf:
                bad.add(r)
                continue
            x = logits[r].double()
            if bool((torch.isnan(x) | (x == math.inf)).any()):
                bad.add(r)
                continue
            z = torch.logsumexp(x * c, 0)
            order = torch.sort(x, descending=True, stable=True).indices[:n_out].tolist()
            for at, t in enumerate(order):
                if float(x[t]) == -math.inf:
                    break
                v = s + float(x[t] * c - z)
                found.append((-v / max(n + 1, 1) ** alpha, b, at, t, v, n + 1))
        found.sort()
        for k in range(n_out):
            f = found[k] if k < len(found) else (0, -1, 0, -1, -math.inf, 0)
            parent.append(f[1]), token.append(f[3]), value.append(f[4]), new_len.append(f[5])
    return parent, token, torch.tensor(value, dtype=torch.float64), new_len, bad


def check_scores(got, want, what=""):
    """Scores rounded once to fp32.  In double they are off by the exponentials' 1.1e-12, by up to 2^18 additions of positive numbers (2^18 2^-53 < 3e-11) in ln Z
    and by a few roundings of numbers below 2^20 (2^-33 each): 1e-9 covers that."""
    got = got.double().cpu()
    assert torch.equal(got == -math.inf, want == -math.inf), what
    fine = want > -math.inf
    off = (got[fine] - want[fine]).abs() - (want[fine].abs() * F32 + 1e-9)
    assert not len(off) or float(off.max()) <= 0, f"{what}: {float(off.max())} beyond the bound"


class PoolModel:
    """rs_page_pool by lists: what each call does to table, counts and pages."""

    def __init__(self, n_slots, max_pages, n_pages, page, k=None, v=None):
        self.table = [[-1] * max_pages for _ in range(n_slots)]
        self.ref = [0] * n_pages
        self.page, self.k, self.v = page, k, v

    def free(self):
        return [p for p, n in enumerate(self.ref) if n == 0]

    def _rows(self, slot, first, end):
        most = self.page * len(self.table[0])
        return [not (0 <= s < len(self.table) and 0 <= a <= b <= most) or s in slot[:i] for i, (s, a, b) in enumerate(zip(slot, first, end))]

    def _is(self, p):
        return 0 <= p < len(self.ref)

    def release(self, slot, first, end):
        bad = self._rows(slot, first, end)
        for s, a, b, wrong in zip(slot, first, end, bad):
            for j in range((a + self.page - 1) // self.page, b // self.page) if not wrong else ():
                if self._is(self.table[s][j]):
                    self.ref[self.table[s][j]] -= 1
                self.table[s][j] = -1
        return [16 * w for w in bad]

    def reserve(self, slot, first, end):
        bad, free, flags, need = self._rows(slot, first, end), self.free(), [], 0
        for s, a, b, wrong in zip(slot, first, end, bad):
            want = [j for j in range(a // self.page, (b + self.page - 1) // self.page) if not self._is(self.table[s][j])] if not wrong and b > a else []
            need += len(want)
            flags.append(16 if wrong else 128 if want and need > len(free) else 0)
            if not flags[-1]:
                for i, j in enumerate(want):
                    p = free[need - len(want) + i]
                    self.table[s][j], self.ref[p] = p, 1
        return flags

    def fork(self, n_beams, slot, parent, pos):
        """(flags, positions)"""
        n, most = len(slot), self.page * len(self.table[0])
        bad = []
        for r in range(n):
            wrong = not 0 <= slot[r] < len(self.table) or slot[r] in slot[:r] or parent[r] >= n_beams
            if not wrong and parent[r] >= 0:
                q = r // n_beams * n_beams + parent[r]
                wrong = not 0 <= slot[q] < len(self.table) or not 0 <= pos[q] <= most
            bad.append(wrong)
        if any(bad):
            return [16 * b for b in bad], None
        table, ref, tails, out_pos = [list(t) for t in self.table], list(self.ref), [], []
        for r in range(n):
            for p in self.table[slot[r]]:
                if self._is(p):
                    ref[p] -= 1
        for r in range(n):
            q = r // n_beams * n_beams + parent[r]
            held = pos[q] if parent[r] >= 0 else 0
            old, whole = self.table[slot[q]], held // self.page
            table[slot[r]] = [p if self._is(p) else -1 for p in old[:whole]] + [-1] * (len(old) - whole)
            for p in table[slot[r]]:
                if p >= 0:
                    ref[p] += 1
            if held % self.page and self._is(old[whole]):
                tails.append((r, whole, old[whole], held % self.page))
            out_pos.append(held)
        copies = []
        for t in tails:
            if ref[t[2]] == 0:
                ref[t[2]] = 1
                table[slot[t[0]]][t[1]] = t[2]
            else:
                copies.append(t)
        free = [p for p, m in enumerate(ref) if m == 0]
        if len(free) < len(copies):
            return [128] * n, None
        for (r, whole, p, tail), to in zip(copies, free):
            table[slot[r]][whole], ref[to] = to, 1
            m = (tail + 7) // 8 * 8
            if self.k is not None:
                self.k[:, to, :, :m], self.v[:, to, :, :, :m] = self.k[:, p, :, :m], self.v[:, p, :, :, :m]
        self.table, self.ref = table, ref
        return [0] * n, out_pos

    def compact(self):
        used = sum(n != 0 for n in self.ref)
        gaps = [p for p in range(used) if self.ref[p] == 0]
        moves = {p: to for p, to in zip([p for p in range(used, len(self.ref)) if self.ref[p]], gaps)}
        for p, to in moves.items():
            self.ref[to], self.ref[p] = self.ref[p], 0
            self.k[:, to], self.v[:, to] = self.k[:, p], self.v[:, p]
        self.table = [[moves.get(p, p) for p in row] for row in self.table]
        return used
