"""Operators below the vocabulary head, and a second loss on it, with their plain forms.

A case is one thing that a training or recognising program does:

  kind "dropout"    dropout of a batch's frames and of their gradient, the mask from a counter-based
                    generator (Philox4x32-10 of Salmon, Moraes, Dror and Shaw, 2011) and never stored;
  kind "embed"      rows of a table by token, scaled (a token below 0 stands for none: zeros);
  kind "embed_grad" the gradient of a table, a row for every class;
  kind "embed_tied" the same added to a gradient that is there (a table that is the head as well);
  kind "ffn"        a gated feed-forward block, act(x Wg^T) * (x Wu^T) Wd^T;
  kind "ffn_train"  the block and its gradients;
  kind "policy"     a clipped policy loss with a KL term on tokens of the head H W^T, with the gradients
                    of H and W (and of the bias).

Element i of a dropout takes the 16-bit half i mod 8 (low half first, word by word) of the four words
that the counter offset + i / 8 and the key seed give; it is kept where that half is below t =
round((1 - p) 65536) and is then multiplied by 65536 / t.  Gradients have the type of what they are gradients of.
Sizes are those of the named workloads and the benchmark, or generic."""
import math

import numpy as np
import torch

own = False

CLIP = (0.2, 0.28)
SEED = 0x1234_5678_9ABC


def _dropout(name, dtype, M, D, p, residual):
    return {"kind": "dropout", "name": name, "dtype": dtype, "M": M, "D": D, "p": p, "residual": residual}


def _embed(name, kind, dtype, out, V, D, N, scale, index="i32", none=0.0):
    return {"kind": kind, "name": name, "dtype": dtype, "out": out, "V": V, "D": D, "N": N, "scale": scale,
            "index": index, "none": none}


def _ffn(name, kind, dtype, M, D, F, act="silu"):
    return {"kind": kind, "name": name, "dtype": dtype, "M": M, "D": D, "F": F, "act": act}


def _policy(name, dtype, M, D, V, bias=False, kl=0.05, none=0.0, old=True, llm=False):
    return {"kind": "policy", "name": name, "dtype": dtype, "M": M, "D": D, "V": V, "bias": bias, "kl": kl,
            "none": none, "old": old, "llm": llm}


def listed():
    return [
        # one utterance's frames before the head: launches count
        _dropout("dropout_utterance", "bf16", 331, 512, 0.1, False),
        # a frozen-head batch's hidden states, dropped and added to the residual stream
        _dropout("dropout_llm", "bf16", 11_458, 4096, 0.1, True),
        # the last labels of 16 utterances' 8 beams, some without a label yet, for a predictor
        _embed("embed_beams", "embed", "f32", "f32", 180_000, 512, 128, math.sqrt(512.0), none=0.1),
        # a batch of transcripts into a language-model table's gradient, a row for every class
        _embed("embed_grad_llm", "embed_grad", "bf16", "bf16", 151_936, 4096, 11_458, 1.0, index="i64"),
        # long text into the gradient that the loss left in the tied head
        _embed("embed_tied", "embed_tied", "bf16", "f32", 151_936, 1024, 65_536, 1.0, none=0.05),
        # a block below the head on one streamed frame
        _ffn("ffn_frame", "ffn", "bf16", 1, 4096, 10_240),
        # one step of 16 utterances' beams
        _ffn("ffn_beams", "ffn", "bf16", 128, 1024, 4096),
        # an encoder's block in fp32 on the benchmark's batch
        _ffn("ffn_train_encoder", "ffn_train", "f32", 4215, 512, 2048, act="gelu"),
        # a language model's block on a training batch
        _ffn("ffn_train_llm", "ffn_train", "bf16", 2567, 4096, 10_240),
        # a short rollout on a small subword head
        _policy("policy_utterance", "bf16", 331, 512, 5000, kl=0.0, old=False),
        # an fp32 head with its bias
        _policy("policy_f32", "f32", 1600, 512, 5000, bias=True, none=0.1),
        # a batch of rollouts on the language-model head, prompts left out
        _policy("policy_llm", "bf16", 2567, 4096, 151_936, none=0.25, llm=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["dropout", "embed", "embed_grad", "embed_tied", "ffn", "ffn_train", "policy", "policy"])
    dtype = "f32" if rng.random() < 0.35 else "bf16"
    wide = 1 if dtype == "bf16" else 2
    if kind == "dropout":
        D = spread(1, 5120)
        c = _dropout("", dtype, spread(1, max(1, 46_000_000 // wide // D)), D, rng.choice([0.0, 0.05, 0.1, 0.3, 0.5, 0.9]),
                     rng.random() < 0.5)
    elif kind in ("embed", "embed_grad", "embed_tied"):
        out = "f32" if dtype == "f32" or (kind == "embed_tied" and rng.random() < 0.7) else "bf16"
        V, D = spread(2, 180_001), spread(1, 4097)
        while V * D > 300_000_000:
            V, D = spread(2, 180_001), spread(1, 4097)
        N = spread(1, min(200_000, max(1, 60_000_000 // D)))
        c = _embed("", kind, dtype, out, V, D, N, rng.choice([1.0, math.sqrt(D), 0.125]), rng.choice(["i32", "i64"]),
                   rng.choice([0.0, 0.1, 0.9]))
    elif kind == "ffn":
        D, F = spread(8, 640) * 8, spread(8, 1280) * 8
        M = spread(1, 4000)
        while M * D * F > 1.2e11 / (wide * wide):
            M = spread(1, 4000)
        c = _ffn("", kind, dtype, M, D, F, rng.choice(["silu", "gelu"]))
    elif kind == "ffn_train":
        D, F = spread(8, 640) * 8, spread(8, 1280) * 8
        M = spread(1, 6000)
        while M * D * F > 1.0e11 / (wide * wide):
            M = spread(1, 6000)
        c = _ffn("", kind, dtype, M, D, F, rng.choice(["silu", "gelu"]))
    else:
        while True:
            D = min(4096, spread(4, 512) * 8)
            V, M = spread(100, 180_001), spread(16, 4500)
            if M * V * D <= (1.2e12 if dtype == "bf16" else 1.2e11):
                break
        c = _policy("", dtype, M, D, V, bias=rng.random() < 0.4, kl=rng.choice([0.0, 0.02, 0.2]),
                    none=rng.choice([0.0, 0.0, 0.3]), old=rng.random() < 0.8, llm=D >= 1024)
    del c["name"]
    return c


# ---- inputs --------------------------------------------------------------------------------

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "i32": torch.int32, "i64": torch.int64}


def _tokens(g, N, V, none):
    """Class ids as text has them: few classes take most of the places (probability about 1 / rank); -1 for none."""
    u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
    rank = torch.exp(u * math.log(V + 1)).long().clamp(1, V) - 1
    ids = (rank * 7919 + 13) % V  # a class's number says little about how common it is
    gone = torch.rand(N, generator=g, device="cuda") < none
    return torch.where(gone, -1, ids)


def prepare(case, seed):
    c = dict(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    dt = TYPES[c["dtype"]]
    x = {"case": c}
    if c["kind"] == "dropout":
        x["x"], x["dy"] = randn(c["M"], c["D"]).to(dt), randn(c["M"], c["D"]).mul_(1e-3).to(dt)
        x["residual"] = randn(c["M"], c["D"]).to(dt) if c["residual"] else None
        x["seed"], x["offset"] = SEED + seed, 10_000_000 * (seed % 1000)
    elif c["kind"].startswith("embed"):
        x["tokens"] = _tokens(g, c["N"], c["V"], c["none"]).to(TYPES[c["index"]])
        if c["kind"] == "embed":
            x["table"] = randn(c["V"], c["D"]).mul_(1 / math.sqrt(c["D"])).to(dt)
        else:
            x["dy"] = randn(c["N"], c["D"]).mul_(1e-3).to(dt)
            if c["kind"] == "embed_tied":
                x["before"] = randn(c["V"], c["D"]).mul_(1e-3).to(TYPES[c["out"]])
                x["dW"] = x["before"].clone()
    elif c["kind"].startswith("ffn"):
        D, F = c["D"], c["F"]
        x["x"] = randn(c["M"], D).to(dt)
        x["wg"], x["wu"] = (randn(F, D).mul_(1 / math.sqrt(D)).to(dt) for _ in range(2))
        x["wd"] = randn(D, F).mul_(1 / math.sqrt(F)).to(dt)
        if c["kind"] == "ffn_train":
            x["dy"] = randn(c["M"], D).mul_(1e-2).to(dt)
    else:
        M, D, V = c["M"], c["D"], c["V"]
        std = 0.02 if c["llm"] else 1.0 / math.sqrt(D)
        W = randn(V, D).mul_(std).to(dt)
        tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
        H = randn(M, D)
        if c["llm"]:
            H /= H.square().mean(1, keepdim=True).sqrt()
        # how far the token's class stands above the rest: from unsure to nearly certain
        lift = torch.rand(M, generator=g, device="cuda") * 8 + math.log(V) - 4
        H += W[tokens].float() * (lift / (D * std * std))[:, None]
        x["H"], x["W"] = H.to(dt), W
        x["bias"] = randn(V).mul_(0.3) if c["bias"] else None
        z = x["H"].float() @ W.float().T
        if c["bias"]:
            z += x["bias"]
        lp = z.gather(1, tokens[:, None])[:, 0] - torch.logsumexp(z, 1)
        del z
        # the policy has moved a little since it sampled: ratios on both sides of the clip's edges, none on them
        moved = randn(M) * 0.2
        for edge in (math.log1p(-CLIP[0]), math.log1p(CLIP[1])):
            moved += torch.where((moved - edge).abs() < 0.01, torch.where(moved < edge, -0.01, 0.01), 0.0)
        x["old"] = lp - moved if c["old"] else None
        x["ref"] = lp + randn(M) * 0.3 if c["kl"] else None
        x["adv"] = randn(M)
        gone = torch.rand(M, generator=g, device="cuda") < c["none"]
        x["tokens"] = torch.where(gone, -1, tokens).int()
        x["weights"] = torch.full((M,), 1.0 / M, device="cuda")
    return x


# ---- plain forms ---------------------------------------------------------------------------

def _philox(counter, seed):
    """Four 32-bit words [n, 4] of each 64-bit counter; all in int64, products by 16-bit halves."""
    low = 0xFFFFFFFF

    def product(m, v):  # high and low 32 bits of m v
        a, b = m * (v & 0xFFFF), m * (v >> 16)
        t = (a >> 16) + (b & low)
        return ((b >> 32 << 16) + (t >> 16)) & low, ((t << 16) | (a & 0xFFFF)) & low

    c0, c1 = counter & low, (counter >> 32) & low
    c2 = c3 = torch.zeros_like(counter)
    for r in range(10):  # (each of the generator's rounds needs the one before)
        k0, k1 = (seed + r * 0x9E3779B9) & low, ((seed >> 32) + r * 0xBB67AE85) & low
        h0, l0 = product(0xD2511F53, c0)
        h1, l1 = product(0xCD9E8D57, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ k0, l1, h0 ^ c3 ^ k1, l0
    return torch.stack([c0, c1, c2, c3], 1)


def _plain_dropout(x, p, seed, offset, residual):
    n = x.numel()
    words = _philox(torch.arange((n + 7) // 8, device=x.device) + offset, seed)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)[:n]
    t = round((1 - p) * 65536)
    y = torch.where(halves < t, x.float().reshape(-1) * (65536 / t), 0.0).view(x.shape)
    return (y if residual is None else y + residual.float()).to(x.dtype)


def _plain_embed(table, tokens, scale):
    y = table[tokens.clamp(min=0).long()].float() * scale
    return torch.where((tokens >= 0)[:, None], y, 0.0).to(table.dtype)


def _plain_embed_grad(dy, tokens, V, scale, before, out):
    live = torch.where(tokens >= 0, tokens, V).long()
    dW = torch.zeros(V + 1, dy.shape[1], device=dy.device)
    dW.index_add_(0, live, dy.float() * scale)
    return (dW[:V] if before is None else before.float() + dW[:V]).to(out)


def _act(a, name):
    return a / (1 + torch.exp(-a)) if name == "silu" else 0.5 * a * (1 + torch.erf(a / math.sqrt(2)))


def _act_grad(a, name):
    if name == "silu":
        s = 1 / (1 + torch.exp(-a))
        return s * (1 + a * (1 - s))
    return 0.5 * (1 + torch.erf(a / math.sqrt(2))) + a * torch.exp(-0.5 * a * a) / math.sqrt(2 * math.pi)


def _plain_ffn(s):
    c = s["case"]
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    a, b = x @ wg.T, x @ wu.T
    h = _act(a, c["act"]) * b
    y = h @ wd.T
    if c["kind"] == "ffn":
        return y.to(s["x"].dtype)
    dy = s["dy"].float()
    dh = dy @ wd
    da, db = dh * b * _act_grad(a, c["act"]), dh * _act(a, c["act"])
    out = {"y": y, "dx": da @ wg + db @ wu, "dw_gate": da.T @ x, "dw_up": db.T @ x, "dw_down": dy.T @ h}
    return {k: v.to(s["x"].dtype) for k, v in out.items()}


def _plain_policy(s):
    c, dt = s["case"], s["H"].dtype
    H, W = s["H"].float(), s["W"].float()
    live = s["tokens"] >= 0
    tok = s["tokens"].clamp(min=0).long()
    z = H @ W.T
    if s["bias"] is not None:
        z += s["bias"]
    top = z.amax(1, keepdim=True)
    lam = (top + torch.log(torch.exp(z - top).sum(1, keepdim=True)))
    lp = torch.where(live, (z.gather(1, tok[:, None]) - lam)[:, 0], 0.0)
    p = torch.exp(z - lam)
    del z
    A = s["adv"]
    r = torch.ones_like(lp) if s["old"] is None else torch.exp(torch.where(live, lp - s["old"], 0.0))
    cut = r.clamp(1 - CLIP[0], 1 + CLIP[1])
    losses = -torch.minimum(r * A, cut * A)
    g = torch.where(r * A <= cut * A, -A * r, 0.0)
    if s["ref"] is not None:
        d = torch.where(live, s["ref"] - lp, 0.0)
        losses = losses + c["kl"] * (torch.exp(d) - d - 1)
        g = g + c["kl"] * (1 - torch.exp(d))
    losses, g = torch.where(live, losses, 0.0), torch.where(live, g * s["weights"], 0.0)
    p *= -g[:, None]
    p[torch.arange(len(g), device=g.device), tok] += g
    out = {"losses": losses, "logp": lp, "dH": (p @ W).to(dt), "dW": (p.T @ H).to(dt)}
    if s["bias"] is not None:
        out["db"] = p.sum(0).to(dt)
    return out


def run(s):
    c = s["case"]
    if own:
        from paper_2609_33645_amd import prunedctc as pc
    if c["kind"] == "dropout":
        if own:
            return {"y": pc.dropout(s["x"], c["p"], s["seed"], s["offset"], residual=s["residual"]),
                    "dx": pc.dropout(s["dy"], c["p"], s["seed"], s["offset"])}
        return {"y": _plain_dropout(s["x"], c["p"], s["seed"], s["offset"], s["residual"]),
                "dx": _plain_dropout(s["dy"], c["p"], s["seed"], s["offset"], None)}
    if c["kind"] == "embed":
        return pc.embedding(s["table"], s["tokens"], c["scale"]) if own else \
            _plain_embed(s["table"], s["tokens"], c["scale"])
    if c["kind"] == "embed_grad":
        return pc.embedding_backward(s["dy"], s["tokens"], c["V"], c["scale"], dtype=TYPES[c["out"]]) if own else \
            _plain_embed_grad(s["dy"], s["tokens"], c["V"], c["scale"], None, TYPES[c["out"]])
    if c["kind"] == "embed_tied":
        if not own:
            return _plain_embed_grad(s["dy"], s["tokens"], c["V"], c["scale"], s["before"], TYPES[c["out"]])
        s["dW"].copy_(s["before"])  # (as the loss's backward would have left it)
        return pc.embedding_backward(s["dy"], s["tokens"], c["V"], c["scale"], out=s["dW"], accumulate=True)
    if c["kind"] == "ffn":
        return pc.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], c["act"])["y"] if own else _plain_ffn(s)
    if c["kind"] == "ffn_train":
        if not own:
            return _plain_ffn(s)
        f = pc.gated_ffn(s["x"], s["wg"], s["wu"], s["wd"], c["act"], keep=True)
        return dict(pc.gated_ffn_backward(s["dy"], s["x"], f["gate"], f["up"], s["wg"], s["wu"], s["wd"], c["act"]),
                    y=f["y"])
    if not own:
        return _plain_policy(s)
    r = pc.policy_loss(s["H"], s["W"], s["tokens"], s["adv"], old_logp=s["old"], ref_logp=s["ref"],
                       weights=s["weights"], bias=s["bias"], clip=CLIP, kl_weight=c["kl"], want_db=c["bias"])
    # (the loss itself is the weighted sum of the losses, which cancel to little more than their roundings)
    return {k: r[k] for k in ("losses", "logp", "dH", "dW") + (("db",) if c["bias"] else ())}


# ---- 64 bits -------------------------------------------------------------------------------

def _exact_kept(n, p, seed, offset):
    """Which of n elements a dropout keeps, from the generator's definition in 64-bit unsigned numbers."""
    u = np.uint64
    low, sh = u(0xFFFFFFFF), u(32)
    ctr = np.arange((n + 7) // 8, dtype=u) + u(offset)
    x = [ctr & low, ctr >> sh, np.zeros_like(ctr), np.zeros_like(ctr)]
    k0, k1 = seed % 2 ** 32, seed >> 32
    for _ in range(10):
        p0, p1 = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(p1 >> sh) ^ x[1] ^ u(k0), p1 & low, (p0 >> sh) ^ x[3] ^ u(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) % 2 ** 32, (k1 + 0xBB67AE85) % 2 ** 32
    w = np.stack(x, 1).astype("<u4").view("<u2").reshape(-1)[:n]
    return torch.from_numpy(w < round((1 - p) * 65536))


def _exact_ffn(s, c):
    x, wg, wu, wd = (s[k].double() for k in ("x", "wg", "wu", "wd"))
    a, b = x @ wg.T, x @ wu.T
    if c["act"] == "silu":
        sg = torch.sigmoid(a)
        f, df = a * sg, sg + a * sg * (1 - sg)
    else:
        phi = 0.5 * torch.erfc(-a * math.sqrt(0.5))
        f, df = a * phi, phi + a * torch.exp(-a * a / 2) / math.sqrt(2 * math.pi)
    y = (f * b) @ wd.T
    if c["kind"] == "ffn":
        return y
    dy = s["dy"].double()
    dh = dy @ wd
    ga, gb = dh * b * df, dh * f
    return {"y": y, "dx": ga @ wg + gb @ wu, "dw_gate": ga.T @ x, "dw_up": gb.T @ x, "dw_down": dy.T @ (f * b)}


def _exact_policy(s, c):
    H, W, A, w = s["H"].double(), s["W"].double(), s["adv"].double(), s["weights"].double()
    M = H.shape[0]
    rows = torch.nonzero(s["tokens"] >= 0)[:, 0]
    tok = s["tokens"][rows].long()
    zero = lambda: torch.zeros(M, dtype=torch.float64, device="cuda")  # noqa: E731
    logp, losses, dH = zero(), zero(), torch.zeros_like(H)
    z = H[rows] @ W.T
    if c["bias"]:
        z += s["bias"].double()
    z -= torch.logsumexp(z, 1, keepdim=True)
    lp = z[torch.arange(len(rows)), tok]
    logp[rows] = lp
    A, w = A[rows], w[rows]
    d = lp - s["old"].double()[rows] if c["old"] else torch.zeros_like(lp)
    ratio = d.exp()
    flat = ((A > 0) & (ratio > 1 + CLIP[1])) | ((A < 0) & (ratio < 1 - CLIP[0]))
    lose = -A * torch.where(flat, torch.where(A > 0, 1 + CLIP[1], 1 - CLIP[0]), ratio)
    coef = torch.where(flat, 0.0, -A * ratio)
    if c["kl"]:
        e = s["ref"].double()[rows] - lp
        lose = lose + c["kl"] * (torch.expm1(e) - e)
        coef = coef - c["kl"] * torch.expm1(e)
    coef = coef * w
    losses[rows] = lose
    z.exp_().mul_(-coef[:, None])
    z[torch.arange(len(rows)), tok] += coef
    dH[rows] = z @ W
    out = {"losses": losses, "logp": logp, "dH": dH, "dW": z.T @ H[rows]}
    if c["bias"]:
        out["db"] = z.sum(0)
    return out


def exact(case, seed):
    c = dict(case)
    s = prepare(c, seed)
    if c["kind"] == "dropout":
        n, t = c["M"] * c["D"], round((1 - c["p"]) * 65536)
        kept = _exact_kept(n, c["p"], s["seed"], s["offset"]).cuda().view(c["M"], c["D"])
        y, dx = (torch.where(kept, s[k].double() * 65536 / t, 0.0) for k in ("x", "dy"))
        return {"y": y if s["residual"] is None else y + s["residual"].double(), "dx": dx}
    if c["kind"] == "embed":
        y = torch.zeros(c["N"], c["D"], dtype=torch.float64, device="cuda")
        live = torch.nonzero(s["tokens"] >= 0)[:, 0]
        y[live] = s["table"][s["tokens"][live].long()].double() * c["scale"]
        return y
    if c["kind"].startswith("embed"):
        live = torch.nonzero(s["tokens"] >= 0)[:, 0]
        dW = torch.zeros(c["V"], c["D"], dtype=torch.float64, device="cuda")
        if c["kind"] == "embed_tied":
            dW += s["before"].double()
        return dW.index_add_(0, s["tokens"][live].long(), s["dy"][live].double(), alpha=c["scale"])
    return _exact_ffn(s, c) if c["kind"].startswith("ffn") else _exact_policy(s, c)


# ---- what a pass cannot do without ---------------------------------------------------------

def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["kind"] == "dropout":
        n = c["M"] * c["D"]
        return {"bytes": e * n * (5 if c["residual"] else 4), "flops": 4 * n}
    if c["kind"].startswith("embed"):
        n, o = c["N"] * c["D"], 4 if c["out"] == "f32" else 2
        ids = c["N"] * (4 if c["index"] == "i32" else 8)
        if c["kind"] == "embed":  # (at most: tokens share rows)
            return {"bytes": e * (min(c["N"], c["V"]) * c["D"] + n) + ids, "flops": n}
        # (the gradient that is there is put in place by the same pass: read once, written once)
        return {"bytes": e * n + ids + o * c["V"] * c["D"] * (2 if c["kind"] == "embed_tied" else 1), "flops": 2 * n}
    if c["kind"].startswith("ffn"):
        M, D, F = c["M"], c["D"], c["F"]
        if c["kind"] == "ffn":
            return {"bytes": e * (2 * M * D + 3 * D * F), "flops": 6 * M * D * F}
        return {"bytes": e * (4 * M * D + 6 * D * F), "flops": 18 * M * D * F}
    M, D, V = c["M"], c["D"], c["V"]
    return {"bytes": 2 * e * D * (M + V) + (4 * V + e * V if c["bias"] else 0) + 24 * M, "flops": 6 * M * D * V}
