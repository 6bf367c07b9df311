"""Oracle of the paged dense cache: plans, and attention over pages, in plain Python and float64.

TEST INFRASTRUCTURE, like the rest of ``oracle/``: only the test suite may use it, and it
shares no code with the GPU library.
"""
from __future__ import annotations

import math

import torch


class Refused(Exception):
    """A step that cannot be planned; the argument is the status it reports."""


class PagePlan:
    """Lengths, tables and the stack of free pages of B requests, a step at a time."""

    def __init__(self, B: int, P: int, n_pages: int, max_pages: int):
        self.P, self.n_pages, self.max_pages = P, n_pages, max_pages
        self.lens = [0] * B
        self.tables = [[] for _ in range(B)]
        self.stack = list(range(n_pages - 1, -1, -1))      # the top is the last

    def step(self, new, keep=None, n_slots=None):
        """(cu, slots) of a step; raises Refused and changes nothing if it cannot be taken."""
        P, B = self.P, len(self.lens)
        kept = [n if keep is None else min(max(keep[b], 0), n) for b, n in enumerate(self.lens)]
        lens = [k + a for k, a in zip(kept, new)]
        pages = [(n + P - 1) // P for n in lens]
        status = 0
        if any(a < 0 for a in new) or sum(len(t) for t in self.tables) + len(self.stack) > self.n_pages:
            status |= 8
        if any(a >= 0 and n > self.max_pages for a, n in zip(new, pages)):
            status |= 2
        if n_slots is not None and (any(a > n_slots for a in new) or (not status and sum(new) > n_slots)):
            status |= 4
        if not status and sum(pages) - sum(len(t) for t in self.tables) > len(self.stack):
            status |= 1
        if status:
            raise Refused(status)
        given = [p for t, n in zip(self.tables, pages) for p in t[n:]]
        tables = [t[:n] for t, n in zip(self.tables, pages)]
        self.stack += reversed(given)
        for t, n in zip(tables, pages):
            while len(t) < n:
                t.append(self.stack.pop())
        self.lens, self.tables = lens, tables
        cu = [sum(new[:b]) for b in range(B + 1)]
        slots = [t[j // P] * P + j % P for t, k, n in zip(tables, kept, lens) for j in range(k, n)]
        return cu, slots + [-1] * ((n_slots if n_slots is not None else len(slots)) - len(slots))


def attention(q, k, v, n_q: int, window: int = 0, sinks: int = 0, scale: float | None = None):
    """Causal attention of a request's last n_q tokens: q [n_q][Hq][d] over k, v [H][L][d].

    Returns out, the weights' mean of |v| (what a relative error of the weights is multiplied by),
    both float64 [n_q][Hq][d], and [n_q][Hq] the largest sum of |q k| over a visible token's
    channels, scaled (what the relative error of a product of d terms is multiplied by).
    """
    Hq, d = q.shape[1:]
    H, L = k.shape[:2]
    scale = 1 / math.sqrt(d) if scale is None else scale
    q, k, v = q.double(), k.double(), v.double()
    pos = torch.arange(L - n_q, L, device=q.device)[:, None]
    j = torch.arange(L, device=q.device)[None]
    sees = j <= pos
    if window:
        sees &= (j > pos - window) | (j < sinks)
    out = torch.zeros((n_q, Hq, d), dtype=torch.float64, device=q.device)
    mean, mag = torch.zeros_like(out), torch.zeros((n_q, Hq), dtype=torch.float64, device=q.device)
    some = sees.any(1)
    if L == 0 or not bool(some.any()):
        return out, mean, mag
    for hq in range(Hq):
        h = hq // (Hq // H)
        s = (q[:, hq] @ k[h].T) * scale
        p = torch.softmax(s.masked_fill(~sees, -math.inf), -1)
        # a token that is not seen takes no part, whatever its value: only products with weights of
        # tokens that are seen are formed
        vh = v[h]
        finite = torch.isfinite(vh)
        o = p.masked_fill(~sees, 0.0) @ torch.where(finite, vh, 0.0)
        for jj in torch.nonzero(~finite.all(1)).flatten().tolist():
            rows = sees[:, jj] & some
            o[rows] += p[rows, jj, None] * torch.where(finite[jj], 0.0, vh[jj])
        out[:, hq] = torch.where(some[:, None], o, 0.0)
        mean[:, hq] = torch.where(some[:, None], p.masked_fill(~sees, 0.0) @ torch.where(finite, vh, 0.0).abs(), 0.0)
        big = (q[:, hq].abs() @ k[h].abs().nan_to_num(0.0, 0.0, 0.0).T) * scale
        mag[:, hq] = big.masked_fill(~sees, 0.0).amax(1)
    return out, mean, mag
