"""Plain 64-bit references of the readout with beams (tests only): candidate classes by their
definition, and prefix beam search on dictionaries keyed by the label tuples themselves."""
from __future__ import annotations

import math
from typing import Dict, List, Sequence, Tuple

import numpy as np

NEG = -math.inf


def logadd(*xs: float) -> float:
    m = max(xs)
    if m == NEG:
        return NEG
    return m + math.log(sum(math.exp(x - m) for x in xs))


def logits(H, W, bias=None) -> np.ndarray:
    z = np.asarray(H, np.float64) @ np.asarray(W, np.float64).T
    return z if bias is None else z + np.asarray(bias, np.float64)


def candidates(z: np.ndarray, C: int, blank: int):
    """ids [M, C] (-1 past the finite logits), logp [M, C], blank_logp [M] of logits z [M, V]."""
    M, V = z.shape
    m = z.max(1, keepdims=True)
    lam = (m + np.log(np.exp(z - m).sum(1, keepdims=True)))[:, 0]
    zz = z.copy()
    zz[:, blank] = NEG
    order = np.argsort(-zz, 1, kind="stable")[:, :C]
    val = np.take_along_axis(zz, order, 1)
    ids = np.full((M, C), -1, np.int64)
    logp = np.full((M, C), NEG)
    k = order.shape[1]
    ids[:, :k] = np.where(val > NEG, order, -1)
    with np.errstate(invalid="ignore"):
        logp[:, :k] = np.where(val > NEG, val - lam[:, None], NEG)
    return ids, logp, z[:, blank] - lam


class Search:
    """One utterance.  gap: the least difference between two totals whose order decided anything."""

    def __init__(self, K: int, bonus: float = 0.0):
        self.K, self.bonus = K, bonus
        self.beams: List[Tuple[tuple, float, float]] = [((), 0.0, NEG)]
        self.gap = math.inf

    def step(self, ids: Sequence[int], logp: Sequence[float], blank: float) -> List[int]:
        score: Dict[int, float] = {int(v): float(l) for v, l in zip(ids, logp) if v >= 0 and l > NEG}
        blank = blank if blank > NEG else NEG
        new: Dict[tuple, list] = {}
        src: Dict[tuple, int] = {}
        rank: Dict[tuple, tuple] = {}
        members = {y for y, _, _ in self.beams}
        for i, (y, pb, pn) in enumerate(self.beams):  # staying
            e = new.setdefault(y, [NEG, NEG])
            e[0] = logadd(e[0], logadd(pb, pn) + blank)
            if y and y[-1] in score:
                e[1] = logadd(e[1], pn + score[y[-1]])
            src[y], rank[y] = i, (0, i, 0)
        for i, (y, pb, pn) in enumerate(self.beams):  # growing
            for r, (v, l) in enumerate(score.items()):
                w = y + (v,)
                e = new.setdefault(w, [NEG, NEG])
                e[1] = logadd(e[1], (pb if y and y[-1] == v else logadd(pb, pn)) + l + self.bonus)
                if w not in members:
                    src[w], rank[w] = i, (1, i, r)
        total = {y: logadd(*e) for y, e in new.items()}
        order = sorted((y for y in new if total[y] > NEG), key=lambda y: (-total[y], rank[y]))
        for a, b in zip(order[:self.K], order[1:self.K + 1]):
            self.gap = min(self.gap, total[a] - total[b])
        keep = order[:self.K]
        self.beams = [(y, new[y][0], new[y][1]) for y in keep]
        return [src[y] for y in keep]

    def run(self, ids, logp, blank) -> "Search":
        for t in range(len(blank)):
            self.step(ids[t], logp[t], blank[t])
        return self

    def result(self):
        return [(y, logadd(pb, pn)) for y, pb, pn in self.beams]
