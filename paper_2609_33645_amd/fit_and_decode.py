"""Fits a CTC head on synthetic speech and reads it out: the training step (Pruned CTC loss and
gradients, clipping by their global norm, update), greedy and beam readout of held-out
utterances, and the same beams as live streams with a predictor state kept per beam.

    python -m paper_2609_33645_amd.fit_and_decode [--steps 300] [--beams 8] [--classes 200]

Every class has a vector; a frame is the vector of the class spoken there plus noise.  The
predictor stands for any state a caller keeps beside a beam (a language model's cache): a
decaying sum of the label vectors of the beam's prefix, advanced when a beam emits labels and
reordered when beams die or branch."""
from __future__ import annotations

import argparse
import json
import sys
from typing import Dict, List

import numpy as np

DECAY = 0.9
SCALE = 3.0  # length of the class vectors


def speak(rng, E: np.ndarray, N: int, noise: float, t_range=(40, 80)):
    """N utterances: frames [M, D], targets, frame counts and label counts (class 0 is blank)."""
    V, D = E.shape
    T = rng.integers(t_range[0], t_range[1] + 1, size=N).astype(np.int32)
    path, targets, U = [], [], []
    for t in T:
        p = np.zeros(t, np.int64)
        at = np.sort(rng.choice(t // 3, size=t // 8, replace=False)) * 3 + 1
        at = at[at < t - 1]
        y = rng.integers(1, V, size=at.size)
        p[at] = y
        held = at[rng.random(at.size) < 0.5]
        p[held + 1] = p[held]
        path.append(p)
        targets.append(y)
        U.append(y.size)
    H = E[np.concatenate(path)] + noise / np.sqrt(D) * rng.standard_normal((int(T.sum()), D))
    return H.astype(np.float32), np.concatenate(targets).astype(np.int32), T, np.array(U, np.int32)


def fit(H, y, T, U, V: int, steps: int, lr: float = 0.2, max_norm: float = 1.0):
    """Head weight and bias (float32) after `steps` updates, and the loss per label and gradient norm
    of every step."""
    import torch

    from . import prunedctc as pc
    D = H.shape[1]
    W = torch.zeros(V, D, device=H.device)
    b = torch.zeros(V, device=H.device)
    momentum = [torch.zeros_like(W), torch.zeros_like(b)]
    weight = torch.full((len(T),), 1.0 / float(U.sum()), device=H.device)
    losses, norms = [], []
    for _ in range(steps):
        out = pc.pruned_ctc_fwd_bwd(H, W, y, T, U, 0, beam=100.0, bias=b, utt_weight=weight, want_dH=False, want_db=True)
        grads = [out["dW"], out["db"]]
        norms.append(pc.clip_grad_norm(grads, max_norm)["norm"])
        for p, m, g in zip((W, b), momentum, grads):
            m.mul_(0.9).add_(g)
            p.sub_(m, alpha=lr)
        losses.append(out["loss"])
    return W, b, torch.cat(losses).cpu().numpy(), torch.cat(norms).cpu().numpy()


def edit_distance(a: List[int], b: List[int]) -> int:
    row = np.arange(len(b) + 1)
    for i, x in enumerate(a, 1):
        prev, row = row, np.empty_like(row)
        row[0] = i
        for j, z in enumerate(b, 1):
            row[j] = min(prev[j] + 1, row[j - 1] + 1, prev[j - 1] + (x != z))
    return int(row[-1])


def stream(H, W, b, T, beams: int, candidates: int, chunk: int, E, token_bonus: float = 0.0):
    """The utterances as live streams, `chunk` frames at a time, each beam with a predictor state
    [N, beams, D].  Returns the result of the search and the states."""
    import torch

    from . import prunedctc as pc
    N = len(T)
    off = np.concatenate([[0], np.cumsum(T)])
    search = pc.BeamSearch(N, beams, int(T.max()), token_bonus)
    state = torch.zeros(N, beams, E.shape[1], device=H.device)
    length = torch.zeros(N, beams, dtype=torch.int32, device=H.device)
    res = search.result(int(T.max()))
    for t in range(0, int(T.max()), chunk):
        counts = np.clip(T - t, 0, chunk)
        rows = np.concatenate([np.arange(off[n] + t, off[n] + t + counts[n]) for n in range(N)])
        c = pc.frame_candidates(H[torch.from_numpy(rows).to(H.device)], W, candidates, 0, b)
        parents = search.advance(c["ids"], c["logp"], c["blank_logp"], counts)
        pc.beam_reorder([state, length], parents)
        res = search.result(int(T.max()))
        for _ in range(chunk):  # labels the beams have gained, one more of each at a time
            grew = length < res["token_lengths"]
            label = res["tokens"].gather(2, length.clamp(max=res["tokens"].shape[2] - 1)[:, :, None].long())[:, :, 0]
            vec = E[torch.where(grew, label, 0).long()]
            state = torch.where(grew[:, :, None], DECAY * state + vec, state)
            length = length + grew.int()
    return res, state


def predictor_of(tokens, lengths, E):
    """The predictor states of finished label sequences, from their definition."""
    import torch
    N, K, L = tokens.shape
    state = torch.zeros(N, K, E.shape[1], device=tokens.device)
    for t in range(L):
        live = (t < lengths)[:, :, None]
        state = torch.where(live, DECAY * state + E[tokens[:, :, t].clamp(min=0).long()], state)
    return state


def run(steps: int = 300, beams: int = 8, classes: int = 200, seed: int = 0, N: int = 12, D: int = 64) -> Dict[str, float]:
    import torch

    from . import prunedctc as pc
    rng = np.random.default_rng(seed)
    E = (SCALE * rng.standard_normal((classes, D)) / np.sqrt(D)).astype(np.float32)
    H, y, T, U = speak(rng, E, 8 * N, noise=1.0)
    dev = torch.device("cuda", torch.cuda.current_device())
    W, b, losses, norms = fit(torch.from_numpy(H).to(dev), torch.from_numpy(y).to(dev), T, U, classes, steps)
    H, y, T, U = speak(rng, E, N, noise=3.0)
    H, Ed = torch.from_numpy(H).to(dev), torch.from_numpy(E).to(dev)
    W, Hb = W.to(torch.bfloat16), H.to(torch.bfloat16)
    C = max(16, beams)
    greedy = pc.greedy_decode(Hb, W, T, 0, b)["tokens"]
    whole = pc.beam_decode(Hb, W, T, beams, C, 0, b)
    live, state = stream(Hb, W, b, T, beams, C, 8, Ed)
    ref = np.split(y, np.cumsum(U)[:-1])
    tokens, lengths = whole["tokens"].cpu().numpy(), whole["token_lengths"].cpu().numpy()
    wrong = {"greedy": 0, "beam": 0, "best of beams": 0}
    for n in range(N):
        errs = [edit_distance(tokens[n, k, :lengths[n, k]].tolist(), ref[n].tolist()) for k in range(beams)
                if lengths[n, k] >= 0]
        wrong["greedy"] += edit_distance(greedy[n], ref[n].tolist())
        wrong["beam"] += errs[0]
        wrong["best of beams"] += min(errs)
    off = float((state - predictor_of(live["tokens"], live["token_lengths"], Ed)).abs().max())
    return {"loss_first": float(losses[0]), "loss_last": float(losses[-1]), "norm_max": float(norms.max()),
            "norm_last": float(norms[-1]), "labels": int(U.sum()), **{f"errors {k}": v for k, v in wrong.items()},
            "streams equal": bool(torch.equal(live["tokens"][:, 0], whole["tokens"][:, 0])),
            "predictor off by": off}


def main(argv=None) -> int:
    ap = argparse.ArgumentParser()
    ap.add_argument("--steps", type=int, default=300)
    ap.add_argument("--beams", type=int, default=8)
    ap.add_argument("--classes", type=int, default=200)
    ap.add_argument("--seed", type=int, default=0)
    a = ap.parse_args(argv)
    r = run(a.steps, a.beams, a.classes, a.seed)
    for k, v in r.items():
        print(f"{k:18s} {v}", flush=True)
    print(json.dumps(r), flush=True)
    return 0


if __name__ == "__main__":
    sys.exit(main())
