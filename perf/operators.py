"""Operators around the vocabulary head's readout and training step, with their plain forms.

A case is one thing that a training or recognising program does:

  kind "clip"     the global norm over a list of gradients, and the clipped gradients in an
                  optimizer's flat buffers;
  kind "reorder"  per-beam state tensors put in the order of the surviving beams;
  kind "stream"   a prefix beam search fed one frame at a time for several streams, a per-beam
                  state (a predictor's) reordered after every frame;
  kind "search"   a prefix beam search over whole utterances, from candidate classes;
  kind "decode"   frames H and head W to the best label sequences: the log probabilities of the
                  most probable classes of every frame over the full vocabulary, then the search.

A search keeps K label prefixes per utterance, each with the log mass of the alignments that end
in blank (pb) and in its last label (pn).  A frame offers blank and C candidate classes; a prefix
stays (blank, or its last label again) or grows by a candidate, the masses of equal prefixes are
added, and the K of largest total are kept (ties: staying prefixes by beam, then grown ones by
beam and candidate).  Sizes are those of the named workloads and the benchmark.
"""
import math

import numpy as np
import torch

own = False

PEAK = 17.0  # nats by which a decoded frame's class stands above the rest


def _clip(name, tensors, **more):
    return dict({"kind": "clip", "name": name, "tensors": tensors, "max_norm": 1.0}, **more)


def _search(name, kind, N, K, C, t_min, t_max, **more):
    return dict({"kind": kind, "name": name, "N": N, "K": K, "C": C, "t_min": t_min, "t_max": t_max, "V": 180_000,
                 "u_frac": 1 / 6, "bonus": 0.0, "state": 0}, **more)


def _decode(name, dtype, D, V, N, K, C, t_min, t_max, **more):
    return dict({"kind": "decode", "name": name, "dtype": dtype, "D": D, "V": V, "N": N, "K": K, "C": C,
                 "t_min": t_min, "t_max": t_max, "u_frac": 1 / 6, "bonus": 0.0, "bias": False, "llm": False}, **more)


def _reorder(name, N, K, rows, width, layers, dtype):
    return {"kind": "reorder", "name": name, "N": N, "K": K, "rows": rows, "width": width, "layers": layers,
            "dtype": dtype}


def listed():
    return [
        # a unit-test sized head and its bias: launches and host work count
        _clip("clip_tiny", "f32:1000x64,f32:1000"),
        # an encoder's many tensors, large and small, some kept in bf16, with the head of 5,000 classes
        _clip("clip_encoder", ",".join(["f32:512x512,bf16:512x2048,f32:512,bf16:2048x512,f32:2048,bf16:33x5x7"] * 60 +
                                       ["f32:5000x512,f32:5000"])),
        # the gradient of the 8B language-model head, beside its input projection's
        _clip("clip_llm_head", "f32:151936x4096,f32:4096x1024,f32:151936"),
        # one utterance's four beams of a small predictor's state
        _reorder("reorder_predictor", 1, 4, 2, 512, 2, "f32"),
        # attention caches of a rescoring language model, 16 utterances of 8 beams
        _reorder("reorder_caches", 16, 8, 375, 1024, 8, "bf16"),
        # one live stream, a frame at a time
        _search("stream_one", "stream", 1, 4, 8, 24, 24, state=512),
        # a serving batch of live streams
        _search("stream_many", "stream", 64, 8, 16, 32, 32, state=1024, bonus=0.3),
        # two long utterances, wide beams
        _search("search_long", "search", 2, 16, 40, 1500, 1500, u_frac=4 / 15),
        # decoding one utterance as it arrives
        _decode("decode_one", "bf16", 512, 180_000, 1, 4, 8, 150, 150),
        # a small subword vocabulary on an fp32 head
        _decode("decode_f32", "f32", 512, 5000, 16, 8, 16, 100, 100, bias=True),
        # the benchmark's batch
        _decode("decode_batch", "bf16", 512, 180_000, 16, 8, 16, 150, 375, bias=True, bonus=-0.3),
        # a batch on the 8B language-model head
        _decode("decode_llm", "bf16", 4096, 151_936, 4, 4, 8, 500, 750, llm=True, u_frac=0.25),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["clip", "reorder", "stream", "search", "decode", "decode"])
    if kind == "clip":
        n = spread(1, 400)
        total = spread(1000, 600_000_000)
        shapes = []
        for _ in range(n):
            w = spread(1, max(1, total // n)) if rng.random() < 0.7 else max(1, total // n)
            shapes.append(f"{rng.choice(['f32', 'bf16'])}:{w}")
        c = _clip("", ",".join(shapes), max_norm=rng.choice([0.5, 1.0, 5.0, 1e9]))
    elif kind == "reorder":
        N, K = spread(1, 64), spread(2, 32)
        width = spread(1, 2048)
        rows = spread(1, max(1, min(2000, 400_000_000 // (N * K * width * 4))))
        c = _reorder("", N, K, rows, width, rng.randint(1, 8), rng.choice(["f32", "bf16"]))
    elif kind in ("stream", "search"):
        K = spread(2, 32)
        C = min(64, max(K, spread(4, 64)))
        N = spread(1, 64 if kind == "stream" else 16)
        t = spread(4, 32) if kind == "stream" else spread(20, 1500)
        c = _search("", kind, N, K, C, max(2, int(t * rng.uniform(0.5, 1.0))), t, V=spread(500, 180_001),
                    u_frac=rng.choice([0.1, 1 / 6, 0.25]), bonus=rng.choice([0.0, 0.0, 0.3, -0.7]),
                    state=spread(1, 1024) if kind == "stream" else 0)
    else:
        while True:
            dtype = "f32" if rng.random() < 0.3 else "bf16"
            step = 8 if rng.random() < 0.3 else 64
            D = min(max(spread(64, 4096) // step * step, 64), 4096)
            V, N, t, K = spread(500, 180_001), spread(1, 32), spread(20, 750), spread(2, 16)
            c = _decode("", dtype, D, V, N, K, min(64, max(K, spread(4, 32))), max(2, int(t * rng.uniform(0.5, 1.0))),
                        t, u_frac=rng.choice([0.1, 1 / 6, 0.25]), bonus=rng.choice([0.0, 0.0, 0.3, -0.7]),
                        bias=rng.random() < 0.4, llm=D >= 1024)
            if int(_lengths(c).sum()) * V * D <= (4e11 if dtype == "bf16" else 1e11):
                break
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------

def _lengths(c):
    r = np.random.default_rng([c["N"], c["t_min"], c["t_max"]])
    return r.integers(c["t_min"], c["t_max"] + 1, size=c["N"]).astype(np.int32)


def _shapes(c):
    for item in c["tensors"].split(","):
        dtype, dims = item.split(":")
        yield (torch.float32 if dtype == "f32" else torch.bfloat16), [int(d) for d in dims.split("x")]


def _transcripts(r, T, u_frac, lo, hi):
    """Per frame, the class that an alignment of a random transcript emits there (-1: blank); labels
    in [lo, hi), lasting one to three frames."""
    path = []
    for t in T:
        p = np.full(t, -1, np.int64)
        for at in np.sort(r.choice(t, size=int(t * u_frac), replace=False)):
            p[at:at + r.integers(1, 4)] = r.integers(lo, hi)
        path.append(p)
    return np.concatenate(path)


def _candidates(c, seed):
    """Candidate classes as a trained head gives them: most frames nearly certain, one in six torn
    between two classes or a class and blank, the others far below."""
    r = np.random.default_rng(seed)
    T = _lengths(c)
    M, C, V = int(T.sum()), c["C"], c["V"]
    half = V // 2
    path = _transcripts(r, T, c["u_frac"], 1, half)
    ids = (r.integers(0, V - 1 - half, size=(M, 1)) + np.arange(C) * ((V - 1 - half) // C)) % (V - 1 - half) + half + 1
    z = -9.0 - np.cumsum(r.exponential(0.4, size=(M, C)), 1)
    blank = np.full(M, -9.0) - r.exponential(1.0, size=M)
    sure = r.exponential(0.3, size=M)
    tok = path >= 0
    blank[~tok] = -sure[~tok]
    ids[tok, 0] = path[tok]
    z[tok, 0] = -sure[tok]
    torn = r.random(M) < 1 / 6
    below = sure + r.uniform(0.3, 6.0, size=M)
    to_blank = torn & tok & (r.random(M) < 0.4)
    blank[to_blank] = -below[to_blank]
    other = torn & ~to_blank
    ids[other, C - 1] = np.where(path[other] >= 0, path[other] % (half - 1) + 1, r.integers(1, half, size=M)[other])
    z[other, C - 1] = -below[other]
    lse = np.log(np.exp(z).sum(1) + np.exp(blank) + 1e-3)
    order = np.argsort(-z, 1, kind="stable")
    ids, z = np.take_along_axis(ids, order, 1), np.take_along_axis(z, order, 1)
    dev = lambda a, t: torch.from_numpy(np.ascontiguousarray(a.astype(t))).cuda()  # noqa: E731
    return T, dev(ids, np.int32), dev(z - lse[:, None], np.float32), dev(blank - lse, np.float32)


def _flat(grads):
    """A buffer per type for the clipped gradients, and each gradient's place in it (an optimizer's
    flat buffers: the places start wherever the sizes before them end)."""
    flat = {}
    for name, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
        n = sum(t.numel() for t in grads if t.dtype == dt)
        if n:
            flat[name] = torch.empty(n, dtype=dt, device="cuda")
    at, out = dict.fromkeys(flat, 0), []
    for t in grads:
        name = "f32" if t.dtype == torch.float32 else "bf16"
        out.append(flat[name][at[name]:at[name] + t.numel()].view(t.shape))
        at[name] += t.numel()
    return flat, out


def _inputs(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = {"case": c}
    if c["kind"] == "clip":
        x["grads"] = [torch.randn(shape, generator=g, device="cuda").mul_(0.02).to(dt) for dt, shape in _shapes(c)]
        x["flat"], x["out"] = _flat(x["grads"])
    elif c["kind"] == "reorder":
        dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
        shape = (c["N"], c["K"], c["rows"], c["width"])
        x["states"] = [torch.randn(shape, generator=g, device="cuda").to(dt) for _ in range(c["layers"])]
        x["out"] = [torch.empty_like(t) for t in x["states"]]
        # survivors descend mostly from the better beams
        u = torch.rand(c["N"], c["K"], generator=g, device="cuda")
        x["parents"] = (u * u * c["K"]).to(torch.int32)
    elif c["kind"] in ("stream", "search"):
        x["T"], x["ids"], x["logp"], x["blank"] = _candidates(c, seed)
        if c["kind"] == "stream":
            # frame t of every stream that still runs, streams in order
            off = np.concatenate([[0], np.cumsum(x["T"])])
            x["steps"] = []
            for t in range(int(x["T"].max())):
                rows = torch.from_numpy(np.array([off[n] + t for n in range(c["N"]) if t < x["T"][n]])).cuda()
                x["steps"].append((x["ids"][rows], x["logp"][rows], x["blank"][rows],
                                   (x["T"] > t).astype(np.int32)))
            x["state"] = torch.randn(c["N"], c["K"], c["state"], generator=g, device="cuda")
            x["spare"] = [torch.empty_like(x["state"]), torch.empty_like(x["state"])]
    else:
        r = np.random.default_rng(seed)
        T = x["T"] = _lengths(c)
        D, V, M = c["D"], c["V"], int(x["T"].sum())
        path = _transcripts(r, T, c["u_frac"], 1, V)
        torn = r.random(M) < 1 / 8
        other = np.where(torn & (path >= 0) & (r.random(M) < 0.4), 0, r.integers(1, V, size=M))
        below = np.where(torn, r.uniform(0.5, 6.0, size=M), np.inf)
        H = torch.randn(M, D, generator=g, device="cuda")
        if c["llm"]:
            H /= H.square().mean(1, keepdim=True).sqrt()
        std = 0.02 if c["llm"] else 1.0 / math.sqrt(D)
        dt = torch.bfloat16 if c["dtype"] == "bf16" else torch.float32
        W = torch.randn(V, D, generator=g, device="cuda").mul_(std).to(dt)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
        add = W[dev(np.maximum(path, 0))].float() * PEAK
        lift = dev(np.maximum(PEAK - below, 0.0).astype(np.float32))
        add += W[dev(other)].float() * lift[:, None]
        H += add / (D * std * std)
        x["H"], x["W"] = H.to(dt), W
        x["bias"] = torch.randn(V, generator=g, device="cuda") * 0.5 if c["bias"] else None
    return x


def prepare(case, seed):
    x = _inputs(dict(case), seed)
    c = x["case"]
    if own and c["kind"] in ("stream", "search"):  # a recogniser keeps its beams' memory
        from paper_2609_33645_amd import prunedctc as pc
        x["beams"] = pc.BeamSearch(c["N"], c["K"], int(x["T"].max()), token_bonus=c["bonus"])
    return x


# ---- plain forms ---------------------------------------------------------------------------

def _plain_clip(grads, max_norm):
    norm = torch.sqrt(sum((g.float() * g.float()).sum() for g in grads))
    scale = torch.clamp(max_norm / (norm + 1e-6), max=1.0)
    flat, out = _flat(grads)
    for g, o in zip(grads, out):
        if g.dtype == torch.float32:
            torch.mul(g, scale, out=o)
        else:
            o.copy_(g.float() * scale)
    return dict(flat, norm=norm.reshape(1))


def _plain_reorder(state, parents):
    N, K = parents.shape
    n = torch.arange(N, device=parents.device)[:, None].expand(N, K)
    return state[n, parents.long()]


class _PlainBeams:
    """Beams as tensors [N, K]: pb and pn (log masses relative to the best prefix), last label,
    number of labels, the labels, and a hash of the labels and of all but the last one."""

    def __init__(self, N, K, L, bonus, dev):
        self.K, self.bonus = K, bonus
        full = lambda v, t: torch.full((N, K), v, dtype=t, device=dev)  # noqa: E731
        self.pb, self.pn = full(-math.inf, torch.float32), full(-math.inf, torch.float32)
        self.pb[:, 0] = 0.0
        self.last, self.len = full(-2, torch.int64), full(0, torch.int64)
        self.hash, self.phash = full(0, torch.int64), full(-1, torch.int64)
        self.tokens = torch.full((N, K, L), -1, dtype=torch.int32, device=dev)
        self.offsets = []
        self.beam = torch.arange(K, device=dev).expand(N, K)

    def step(self, live, ids, lp, bl):
        """One frame of the utterances `live` [N] (ids, lp [N, C] and bl [N]: any values elsewhere);
        returns the beam that each new one descends from."""
        K, inf = self.K, math.inf
        N, C = ids.shape
        ids = ids.long()
        s = torch.logaddexp(self.pb, self.pn)
        lb = lp + self.bonus
        same = self.last[:, :, None] == ids[:, None, :]
        lp_last = torch.where(same, lp[:, None, :], -inf).amax(2)
        ext = torch.where(same, self.pb[:, :, None], s[:, :, None]) + lb[:, None, :]
        # merge[n, i, j]: prefix i grown by j's last label is prefix j
        alive = s > -inf
        merge = (self.phash[:, None, :] == self.hash[:, :, None]) & (self.len[:, None, :] == self.len[:, :, None] + 1)
        merge &= alive[:, None, :] & alive[:, :, None]
        base = torch.where(self.last[:, :, None] == self.last[:, None, :], self.pb[:, :, None], s[:, :, None])
        lb_last = torch.where(same, lb[:, None, :], -inf).amax(2)
        add = torch.where(merge, base + lb_last[:, None, :], -inf).amax(1)
        taken = (merge[:, :, :, None] & same[:, None, :, :]).any(2)
        ext = torch.where(taken, -inf, ext)
        stay_b = s + bl[:, None]
        stay_n = torch.logaddexp(self.pn + lp_last, add)
        total = torch.cat([torch.logaddexp(stay_b, stay_n), ext.reshape(N, K * C)], 1)
        val, idx = torch.sort(total, dim=1, descending=True, stable=True)
        val, idx = val[:, :K], idx[:, :K]
        grown = idx >= K
        par = torch.where(grown, (idx - K) // C, idx)
        tok = torch.gather(ids, 1, (idx - K).clamp(min=0) % C)
        pick = lambda a: torch.gather(a, 1, par)  # noqa: E731
        best = val[:, :1]
        pb = torch.where(grown, -inf, pick(stay_b)) - best
        pn = torch.where(grown, val, pick(stay_n)) - best
        ln, hs = pick(self.len), pick(self.hash)
        tokens = torch.gather(self.tokens, 1, par[:, :, None].expand_as(self.tokens))
        at = torch.where(grown, ln, self.tokens.shape[2] - 1)[:, :, None]
        tokens.scatter_(2, at, torch.where(grown, tok, tokens[:, :, -1].long()).int()[:, :, None])
        keep = live[:, None]
        upd = lambda new, old: torch.where(keep, new, old)  # noqa: E731
        self.phash = upd(torch.where(grown, hs, pick(self.phash)), self.phash)
        self.hash = upd(torch.where(grown, (hs ^ (tok + 1)) * 0x5851F42D4C957F2D + 0x14057B7EF767814F, hs), self.hash)
        self.last = upd(torch.where(grown, tok, pick(self.last)), self.last)
        self.len = upd(ln + grown, self.len)
        self.pb, self.pn = upd(pb, self.pb), upd(pn, self.pn)
        self.tokens = torch.where(keep[:, :, None], tokens, self.tokens)
        self.offsets.append(torch.where(live, best[:, 0], 0.0))
        return torch.where(keep, par, self.beam).int()

    def result(self):
        score = torch.logaddexp(self.pb, self.pn) + torch.stack(self.offsets).sum(0)[:, None]
        return {"tokens": self.tokens, "token_lengths": self.len.int(), "scores": score}


def _padded(T, packed):
    """Frames packed utterance after utterance as [T_max, N, ...] (the last frame repeated)."""
    off = np.concatenate([[0], np.cumsum(T)])[:-1]
    at = torch.from_numpy(off[None, :] + np.minimum(np.arange(T.max())[:, None], T[None, :] - 1)).cuda()
    return packed[at]


def _plain_search(c, T, ids, logp, blank):
    beams = _PlainBeams(c["N"], c["K"], int(T.max()), c["bonus"], ids.device)
    ids, logp, blank = _padded(T, ids), _padded(T, logp), _padded(T, blank)
    live = torch.from_numpy(np.arange(T.max())[:, None] < T[None, :]).cuda()
    for t in range(int(T.max())):
        beams.step(live[t], ids[t], logp[t], blank[t])
    return beams.result()


def _plain_stream(s):
    c, T = s["case"], s["T"]
    beams = _PlainBeams(c["N"], c["K"], int(T.max()), c["bonus"], s["ids"].device)
    ids, logp, blank = _padded(T, s["ids"]), _padded(T, s["logp"]), _padded(T, s["blank"])
    live = torch.from_numpy(np.arange(T.max())[:, None] < T[None, :]).cuda()
    state, parents = s["state"], []
    for t in range(int(T.max())):
        parents.append(beams.step(live[t], ids[t], logp[t], blank[t]))
        state = _plain_reorder(state, parents[-1])
    return dict(beams.result(), parents=torch.stack(parents), state=state)


def _plain_candidates(H, W, bias, C):
    z = H.float() @ W.float().T
    if bias is not None:
        z += bias
    top = z.amax(1)
    lam = top + torch.log(torch.exp(z - top[:, None]).sum(1))
    blank = z[:, 0] - lam
    z[:, 0] = -math.inf
    val, idx = torch.topk(z, C, 1)
    idx, order = torch.sort(idx, 1)
    val, order = torch.sort(torch.gather(val, 1, order), dim=1, descending=True, stable=True)
    return torch.gather(idx, 1, order).int(), val - lam[:, None], blank


def run(s):
    c = s["case"]
    if c["kind"] == "clip":
        if own:
            from paper_2609_33645_amd import prunedctc as pc
            r = pc.clip_grad_norm(s["grads"], c["max_norm"], out=s["out"])
            return dict(s["flat"], norm=r["norm"])
        return _plain_clip(s["grads"], c["max_norm"])
    if c["kind"] == "reorder":
        if own:
            from paper_2609_33645_amd import prunedctc as pc
            return pc.beam_reorder(s["states"], s["parents"], out=s["out"])
        return [_plain_reorder(t, s["parents"]) for t in s["states"]]
    if c["kind"] == "stream":
        if not own:
            return _plain_stream(s)
        from paper_2609_33645_amd import prunedctc as pc
        b = s["beams"]
        b.reset()
        state, parents = s["state"], []
        for i, (ids, logp, blank, counts) in enumerate(s["steps"]):
            parents.append(b.advance(ids, logp, blank, counts))
            state = pc.beam_reorder([state], parents[-1], out=[s["spare"][i % 2]])[0]
        return dict(b.result(), parents=torch.stack(parents), state=state)
    if c["kind"] == "search":
        if not own:
            return _plain_search(c, s["T"], s["ids"], s["logp"], s["blank"])
        b = s["beams"]
        b.reset()
        b.advance(s["ids"], s["logp"], s["blank"], s["T"])
        return b.result()
    if own:
        from paper_2609_33645_amd import prunedctc as pc
        r = pc.beam_decode(s["H"], s["W"], s["T"], beam_size=c["K"], candidates=c["C"], bias=s["bias"],
                           token_bonus=c["bonus"])
        return {k: r[k] for k in ("tokens", "token_lengths", "scores", "logp", "blank_logp")}
    ids, logp, blank = _plain_candidates(s["H"], s["W"], s["bias"], c["C"])
    return dict(_plain_search(c, s["T"], ids, logp, blank), logp=logp, blank_logp=blank)


# ---- 64 bits -------------------------------------------------------------------------------

def _logadd(a, b):
    if a < b:
        a, b = b, a
    return a if b == -math.inf else a + math.log1p(math.exp(b - a))


def _exact_step(beams, K, bonus, ids, lp, blank):
    """beams: list of (labels, pb, pn), best first.  Returns the next list and the positions in
    `beams` that its members come from."""
    at = {y: i for i, (y, _, _) in enumerate(beams)}
    score = dict(zip(ids, lp))
    total = [_logadd(pb, pn) for _, pb, pn in beams]
    taken = [set() for _ in beams]  # labels by which a beam would grow into another beam
    new = []
    for i, (y, pb, pn) in enumerate(beams):
        p = -math.inf
        j = at.get(y[:-1]) if y else None
        if j is not None:
            taken[j].add(y[-1])
        if y and y[-1] in score:
            p = pn + score[y[-1]]
            if j is not None:
                before = beams[j][1] if beams[j][0] and beams[j][0][-1] == y[-1] else total[j]
                p = _logadd(p, before + score[y[-1]] + bonus)
        new.append((_logadd(total[i] + blank, p), i, None, total[i] + blank, p))
    for i, (y, pb, pn) in enumerate(beams):
        last = y[-1] if y else None
        for v, l in score.items():
            if v not in taken[i]:
                p = (pb if v == last else total[i]) + l + bonus
                new.append((p, i, v, -math.inf, p))
    new.sort(key=lambda e: -e[0])
    new = new[:K]
    return [(beams[i][0] + (() if v is None else (v,)), b, p) for _, i, v, b, p in new], [e[1] for e in new]


def _exact_result(all_beams, L):
    N, K = len(all_beams), len(all_beams[0])
    tokens = np.full((N, K, L), -1, np.int32)
    for n, beams in enumerate(all_beams):
        for k, (y, _, _) in enumerate(beams):
            tokens[n, k, :len(y)] = y
    return {"tokens": torch.from_numpy(tokens),
            "token_lengths": torch.tensor([[len(y) for y, _, _ in b] for b in all_beams], dtype=torch.int32),
            "scores": torch.tensor([[_logadd(pb, pn) for _, pb, pn in b] for b in all_beams], dtype=torch.float64)}


def _exact_search(c, T, ids, logp, blank):
    off = np.concatenate([[0], np.cumsum(T)])
    out, parents = [], np.tile(np.arange(c["K"], dtype=np.int32), (int(T.max()), c["N"], 1))
    for n in range(c["N"]):
        beams = [((), 0.0, -math.inf)]
        for t in range(T[n]):
            m = off[n] + t
            beams, src = _exact_step(beams, c["K"], c["bonus"], ids[m], logp[m], blank[m])
            parents[t, n] = src
        out.append(beams)
    return _exact_result(out, int(T.max())), parents


def exact(case, seed):
    c = dict(case)
    if c["kind"] in ("stream", "search", "decode") and \
            int(_lengths(c).sum()) * c["K"] * (c["C"] + 4) > 5_000_000:
        return None
    x = _inputs(c, seed)
    if c["kind"] == "clip":
        norm = math.sqrt(sum(float(t.double().square().sum()) for t in x["grads"]))
        scale = min(1.0, c["max_norm"] / (norm + 1e-6))
        r = {"norm": torch.tensor([norm], dtype=torch.float64)}
        for name, dt in (("f32", torch.float32), ("bf16", torch.bfloat16)):
            if name in x["flat"]:
                r[name] = torch.cat([t.double().reshape(-1) * scale for t in x["grads"] if t.dtype == dt])
        return r
    if c["kind"] == "reorder":
        p = x["parents"].tolist()
        return [torch.stack([torch.stack([t[n, k] for k in p[n]]) for n in range(c["N"])]) for t in x["states"]]
    if c["kind"] == "decode":
        ids, logp, blank = [], [], []
        W = x["W"].double().T
        for m in range(0, x["H"].shape[0], 512):
            z = x["H"][m:m + 512].double() @ W
            if x["bias"] is not None:
                z += x["bias"].double()
            lam = torch.logsumexp(z, 1)
            blank += (z[:, 0] - lam).tolist()
            val, idx = torch.topk(z[:, 1:], c["C"], 1)
            ids += (idx + 1).tolist()
            logp += (val - lam[:, None]).tolist()
        f64 = lambda a: torch.tensor(a, dtype=torch.float64)  # noqa: E731
        return dict(_exact_search(c, x["T"], ids, logp, blank)[0], logp=f64(logp), blank_logp=f64(blank))
    r, parents = _exact_search(c, x["T"], x["ids"].tolist(), x["logp"].tolist(), x["blank"].tolist())
    if c["kind"] == "search":
        return r
    state, steps = x["state"].cpu(), torch.from_numpy(parents)
    for p in steps:
        state = torch.stack([state[n][p[n].long()] for n in range(c["N"])])
    return dict(r, parents=steps, state=state)


# ---- what a pass cannot do without ---------------------------------------------------------

def work(case):
    c = case
    if c["kind"] == "clip":
        n = b = 0
        for dt, shape in _shapes(c):
            k = math.prod(shape)
            n += k
            b += k * (4 if dt == torch.float32 else 2)
        return {"bytes": 2 * b, "flops": 3 * n}
    if c["kind"] == "reorder":
        b = c["N"] * c["K"] * c["rows"] * c["width"] * c["layers"] * (4 if c["dtype"] == "f32" else 2)
        return {"bytes": 2 * b + 4 * c["N"] * c["K"], "flops": 0}
    M = int(_lengths(c).sum())
    K, C, L = c["K"], c["C"], int(_lengths(c).max())
    out = c["N"] * K * (4 * L + 8)
    step = M * K * (C + 8) * 4
    if c["kind"] in ("stream", "search"):
        return {"bytes": M * (8 * C + 4) + out + 2 * 4 * M * K * c["state"], "flops": step}
    e = 4 if c["dtype"] == "f32" else 2
    return {"bytes": e * c["D"] * (M + c["V"]) + (4 * c["V"] if c["bias"] else 0) + out + 4 * M * (C + 1),
            "flops": 2 * M * c["V"] * c["D"] + step}
