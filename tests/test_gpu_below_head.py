"""Dropout, token embedding, the gated block and the policy loss on the GPU, against 64-bit references
(all through the public binding).

A rounding is off by at most half a step: 2^-24 of the value in float32, 2^-8 in bfloat16 (E below)."""
import math

import numpy as np
import pytest

from tests import below_head_ref as ref
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

F = 2.0 ** -24
E = {"bf16": 2.0 ** -8, "f32": F}


def kind(dtype):
    import torch
    return {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to(kind(dtype)) if dtype else t


def host(t):
    return t.double().cpu().numpy()


def within(got, want, tol, what=""):
    got = host(got)
    assert got.shape == want.shape, (got.shape, want.shape)
    assert np.isfinite(got).all(), what
    d = np.abs(got - want)
    bad = d > tol
    assert not bad.any(), (what, int(bad.sum()), d[bad].max(), np.broadcast_to(tol, d.shape)[bad].min(), np.argwhere(bad)[:4])


# ---- dropout -------------------------------------------------------------------------------

def check_dropout(x, got, p, seed, offset, residual=None):
    """The scale is rounded to float, the product (or the sum with the residual) once more, and the
    result once to its type."""
    dtype = "f32" if x.element_size() == 4 else "bf16"
    r = None if residual is None else host(residual)
    want = ref.dropout(host(x), p, seed, offset, r)
    part = np.abs(ref.dropout(host(x), p, seed, offset))
    within(got, want, part * (2 * F) + np.abs(want) * (F + E[dtype]) + 1e-38, (dtype, p))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [0, 1, 7, 8, 9, 4095, 4096, 4097, 8191, 100_003])
@pytest.mark.parametrize("p,residual", [(0.0, False), (0.1, True), (0.5, False), (0.9, True), (1 - 2.0 ** -16, False)])
def test_dropout(dtype, n, p, residual):
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("dropout", dtype, n, p, residual)
    g = torch.Generator().manual_seed(n + 1)
    x = torch.randn(n, generator=g).cuda().to(kind(dtype))
    r = torch.randn(n, generator=g).cuda().to(kind(dtype)) if residual else None
    seed, offset = 0xFEDC_BA98_7654_3210 ^ n, (1 << 33) + 5
    got = pc.dropout(x, p, seed, offset, residual=r)
    check_dropout(x, got, p, seed, offset, r)
    if p == 0.0:
        assert torch.equal(got, x)
    # in place, and into the residual
    y = x.clone()
    assert pc.dropout(y, p, seed, offset, residual=r, out=y) is y and torch.equal(y, got)
    if residual:
        z = r.clone()
        assert torch.equal(pc.dropout(x, p, seed, offset, residual=z, out=z), got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dropout_views_shapes_and_counters(dtype):
    """Values at any alignment and layout; the mask goes by place and counters, whatever the call."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("dropout views", dtype)
    flat = torch.randn(5003).cuda().to(kind(dtype))
    for a in (1, 2, 3, 5):
        x = flat[a:a + 4001]
        buf = torch.full((5003,), 7.0, device="cuda", dtype=kind(dtype))
        pc.dropout(x, 0.3, 11, 2 ** 64 - 3, out=buf[a + 1:a + 4002])  # (the counter wraps)
        check_dropout(x, buf[a + 1:a + 4002], 0.3, 11, 2 ** 64 - 3)
        assert (buf[:a + 1] == 7).all() and (buf[a + 4002:] == 7).all()
    x = torch.randn(33, 5, 7, device="cuda").to(kind(dtype))
    y = pc.dropout(x.transpose(0, 2), 0.4, 3)
    assert y.shape == (7, 5, 33)
    check_dropout(x.transpose(0, 2).contiguous(), y, 0.4, 3, 0)
    # consecutive calls use consecutive counters
    x = torch.randn(64, 40, device="cuda").to(kind(dtype))
    whole = pc.dropout(x, 0.5, 9, 100)
    parts = [pc.dropout(x[i:i + 16], 0.5, 9, 100 + i * 5) for i in range(0, 64, 16)]
    assert torch.equal(whole, torch.cat(parts))
    # a dropped value that is not finite is zero, a kept one stays
    x = torch.full((1000,), math.inf, device="cuda", dtype=kind(dtype))
    y = pc.dropout(x, 0.5, 1)
    k = dev(ref.kept(1000, 0.5, 1, 0))
    assert torch.equal(y, torch.where(k, x, torch.zeros_like(x)))


def test_dropout_counter_on_the_device_in_a_graph():
    """A captured call reads its counter at each replay; other work and synchronizations between."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("dropout graph")
    x = torch.randn(777, 65, device="cuda")
    counter = torch.zeros(1, dtype=torch.int64, device="cuda")
    y = torch.empty_like(x)
    pc.dropout(x, 0.2, 5, counter, out=y)  # (the library is loaded before a capture)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pc.dropout(x, 0.2, 5, counter, out=y)
        counter += (x.numel() + 7) // 8
    for i in range(4):
        g.replay()
        at = i * ((x.numel() + 7) // 8)
        assert torch.equal(y, pc.dropout(x, 0.2, 5, at)), i
        torch.cuda.synchronize()
        x.normal_()


# ---- embedding -----------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V,D,N", [(1, 1, 1), (2, 3, 7), (5, 8, 0), (7, 9, 65), (1000, 33, 300), (257, 512, 128), (300, 4097, 5),
                                   (180_001, 4, 2000)])
@pytest.mark.parametrize("wide", [False, True])
def test_embedding(dtype, V, D, N, wide):
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("embedding", dtype, V, D, N, wide)
    r = np.random.default_rng(V + D)
    table = dev(r.normal(size=(V, D)).astype(np.float32), dtype)
    t = r.integers(-1, V + 1, size=N)
    if wide and N:
        t[:: 3] += 2 ** 32  # (classes once cut to 32 bits)
    tokens = torch.from_numpy(t).cuda().to(torch.int64 if wide else torch.int32)
    for scale in (1.0, -0.3):
        want = ref.embedding(host(table), t, float(np.float32(scale)))
        within(pc.embedding(table, tokens, scale), want, np.abs(want) * (F + E[dtype]), scale)
    if N >= 6:
        shaped = pc.embedding(table, tokens[:6].view(2, 3))
        assert shaped.shape == (2, 3, D) and torch.equal(shaped.view(6, D), pc.embedding(table, tokens[:6]))


def check_grad(dy, t, V, scale, got, before=None):
    """A class's n rows summed in float, in any order: at most n roundings of a partial sum each, which is no
    larger than the sum of magnitudes; the scale's and the result's roundings, and one of the sum with
    what was there."""
    want, mag, n = ref.embedding_backward(host(dy), t, V, float(np.float32(scale)))
    dtype = "f32" if got.element_size() == 4 else "bf16"
    tol = mag * (F * (n[:, None] + 2))
    if before is not None:
        want = want + before
    within(got, want, tol + np.abs(want) * (F + E[dtype]), (dtype, V, len(t)))


@pytest.mark.parametrize("V,D,N", [(1, 1, 1), (1, 5, 40), (3, 8, 7), (4, 9, 8), (5, 16, 9), (100, 33, 64), (100, 64, 65), (90, 24, 1023),
                                   (2000, 40, 1024), (700, 2049, 130), (5000, 8, 15_360), (5000, 9, 15_361), (5000, 8, 16_384), (5000, 12, 16_385), (180_001, 3, 40_000),
                                   (500, 4, 70_000), (524_288, 1, 33_000)])
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_embedding_backward(V, D, N, dtype, out):
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("embedding_backward", V, D, N, dtype, out)
    r = np.random.default_rng(V * 3 + N)
    # common classes, rare ones and places without a token
    t = np.minimum((r.random(N) ** 3 * (V + 1)).astype(np.int64), V) - (r.random(N) < 0.1) * (V + 5)
    dy = dev(r.normal(size=(N, D)).astype(np.float32), dtype)
    tokens = torch.from_numpy(t).cuda().int()
    got = pc.embedding_backward(dy, tokens, V, 0.7, dtype=kind(out))
    check_grad(dy, t, V, 0.7, got)
    again = pc.embedding_backward(dy, tokens.long(), V, 0.7, out=torch.full((V, D), math.nan, device="cuda", dtype=kind(out)))
    assert torch.equal(got, again)
    # added to what is there; rows without a token are left as they are
    base = torch.randn(V, D, device="cuda").to(kind(out))
    acc = pc.embedding_backward(dy, tokens, V, 0.7, out=base.clone(), accumulate=True)
    check_grad(dy, t, V, 0.7, acc, host(base))
    idle = np.setdiff1d(np.arange(V), t)
    idle = torch.from_numpy(idle).cuda()
    assert torch.equal(acc[idle], base[idle])


@pytest.mark.parametrize("N", [5, 500, 3000, 20_000])
@pytest.mark.parametrize("which", ["one class", "none", "two", "edges"])
def test_embedding_backward_of_few_classes(N, which):
    """All tokens of one class (its sum crosses every range), of none, of two in blocks, of the first and last."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("embedding_backward few", N, which)
    V, D = 300, 20
    t = {"one class": np.full(N, 17), "none": np.full(N, -1), "two": np.where(np.arange(N) < N // 3, 200, 3),
         "edges": np.where(np.arange(N) % 5 == 0, 0, V - 1)}[which]
    dy = dev(np.random.default_rng(N).normal(size=(N, D)).astype(np.float32), "bf16")
    tokens = torch.from_numpy(t).cuda()
    got = pc.embedding_backward(dy, tokens, V, dtype=torch.float32)
    check_grad(dy, t, V, 1.0, got)


def test_embedding_backward_of_a_view_and_in_a_graph():
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("embedding_backward view, graph")
    buf = torch.randn(50, 200, device="cuda")
    t = torch.arange(50, device="cuda") % 7
    out = torch.full((9 * 13 + 3,), 5.0, device="cuda")
    view = out[1:1 + 9 * 13].view(9, 13)
    pc.embedding_backward(buf[:, 3:16], t, 9, out=view)  # rows with a stride; a result that starts anywhere
    check_grad(buf[:, 3:16].contiguous(), t.cpu().numpy(), 9, 1.0, view)
    assert out[0] == 5 and (out[1 + 9 * 13:] == 5).all()
    # Two graphs with memory of their own, replayed in turn with eager calls between
    graphs = []
    for n in (300, 20_000):
        dy, tok = torch.randn(n, 33, device="cuda"), torch.randint(0, 400, (n,), device="cuda")
        dW = torch.empty(400, 33, device="cuda")
        pc.embedding_backward(dy, tok, 400, out=dW)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pc.embedding_backward(dy, tok, 400, out=dW)
        graphs.append((g, dy, tok, dW))
    for i in range(3):
        for g, dy, tok, dW in graphs:
            dy.normal_()
            tok.copy_(torch.randint(-1, 401, tok.shape, device="cuda"))
            g.replay()
            assert torch.equal(dW, pc.embedding_backward(dy, tok, 400)), i
        torch.cuda.synchronize()


# ---- policy loss ---------------------------------------------------------------------------

def policy_case(seed, M, D, V, dtype, bias=False, sure=4.0, clip=(0.2, 0.3)):
    """H, W, bias, tokens (some left out), advantages, old and reference log probabilities (no ratio within
    1e-3 of the clip's edges), weights."""
    r = np.random.default_rng(seed)
    W = r.normal(size=(V, D)) / math.sqrt(D)
    t = r.integers(0, V, size=M)
    H = r.normal(size=(M, D)) + W[t] * (r.random((M, 1)) * 2 * sure + math.log(V) - sure)
    H, W = (host(dev(x.astype(np.float32), dtype)) for x in (H, W))
    b = (r.normal(size=V) * 0.3).astype(np.float32) if bias else None
    z = H @ W.T + (0 if b is None else b)
    top = z.max(1)
    lp = z[np.arange(M), t] - top - np.log(np.exp(z - top[:, None]).sum(1))
    moved = r.normal(size=M) * 0.2
    for edge in (math.log(1 - clip[0]), math.log(1 + clip[1])):
        near = np.abs(moved - edge) < 1e-3
        moved[near] += 3e-3
    t = np.where(r.random(M) < 0.15, r.choice([-1, V, -7], size=M), t)
    f = lambda x: x.astype(np.float32)  # noqa: E731
    return dict(H=H, W=W, bias=b, tokens=t, adv=f(r.normal(size=M)), old=f(lp - moved), ref=f(lp + r.normal(size=M) * 0.5),
                w=f(r.random(M) + 0.5))


def policy_call(c, dtype, clip, kl, **kw):
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    d = lambda x: None if x is None else dev(x)  # noqa: E731
    return pc.policy_loss(dev(c["H"].astype(np.float32), dtype), dev(c["W"].astype(np.float32), dtype),
                          torch.from_numpy(c["tokens"]).cuda().int(), d(c["adv"]), d(c["old"]), d(c["ref"]), d(c["w"]),
                          d(c["bias"]), clip=clip, kl_weight=kl, **kw)


def check_policy(c, dtype, clip, kl, got, db=False, status=None, own_rounded=True):
    """Errors to first order.  A logit: (D + 2) 2^-24 of the sum of its terms' magnitudes; lambda: the largest logit's
    error and 2e-5, the normaliser's bar.  From these the token's log probability (one rounding more), its
    ratio and KL factor, hence g; a probability by its logit's and lambda's errors and the exponential's
    2^-21; dZ by these and one rounding to the products' type (of the token's own entry: of g (1 - p), whose p
    is off by the log probability's error).  Products: magnitudes times the roundings of their sums, at most one
    per 16 terms on the matrix cores and one per slice, taken as one per term; a rounding at the end.
    float32 products drop 2^-24 of each term and round six times per 16 terms: the same bound.
    own_rounded False: the rounding of the tokens' own entries is made good in the gradients."""
    lo, hi = clip
    w = ref.policy(c["H"], c["W"], c["bias"], c["tokens"], c["adv"], c["old"], c["ref"], c["w"], lo, hi, kl)
    M, V = w["p"].shape
    D = c["H"].shape[1]
    mass = np.abs(c["H"]) @ np.abs(c["W"]).T + (0 if c["bias"] is None else np.abs(c["bias"]))
    ez = (D + 2) * F * mass
    el = ez.max(1) + 2e-5
    ok = (c["tokens"] >= 0) & (c["tokens"] < V)
    t = np.where(ok, c["tokens"], 0)
    elp = np.where(ok, ez[np.arange(M), t] + el + F * np.abs(w["logp"]), 0.0)
    if status is None:
        within(got["logp"], w["logp"], elp, "logp")
    assert (got["status"].cpu().numpy() == (np.where(ok, 0, 1) if status is None else status)).all()
    A = np.abs(c["adv"].astype(np.float64))
    r = np.ones(M) if c["old"] is None else np.exp(w["logp"] - c["old"])
    x = np.zeros(M) if c["ref"] is None else np.exp(c["ref"] - w["logp"])
    eloss = np.where(ok, (A * r + kl * (x + 1)) * elp * 1.01 + 2 * F * np.abs(w["losses"]), 0.0)
    within(got["losses"], w["losses"], eloss, "losses")
    wt = np.ones(M) if c["w"] is None else c["w"].astype(np.float64)
    within(got["loss"], np.array([w["loss"]]), (eloss * wt).sum() + 1e-12, "loss")
    eg = np.where(ok, wt * (A * r + kl * x) * elp * 1.01, 0.0) + 2 * F * np.abs(w["g"])
    g = np.abs(w["g"])[:, None]
    e = E["bf16"] if dtype == "bf16" else F
    ep = w["p"] * ((ez + el[:, None]) * 1.01 + 2.0 ** -21)
    edz = g * ep + eg[:, None] * w["p"] + e * np.abs(w["dZ"])
    rows = np.nonzero(ok)[0]
    own = (rows, t[rows])
    edz[own] = (g[rows, 0] * w["p"][own] * elp[rows] * 1.01 + eg[rows] * (1 - w["p"][own])
                + ((e if own_rounded else 0) + 4 * F) * np.abs(w["dZ"][own]))
    dz = np.abs(w["dZ"]) + edz
    aW, aH = np.abs(c["W"]), np.abs(c["H"])
    out = E[dtype]
    tiny = 1e-37
    within(got["dH"], w["dH"], edz @ aW + (V + 8) * F * (dz @ aW) + out * np.abs(w["dH"]) * 1.01 + tiny, "dH")
    within(got["dW"], w["dW"], edz.T @ aH + (M + 8) * F * (dz.T @ aH) + out * np.abs(w["dW"]) * 1.01 + tiny, "dW")
    if db:
        within(got["db"], w["db"], edz.sum(0) + (M + 8) * F * dz.sum(0) + out * np.abs(w["db"]) * 1.01 + tiny, "db")
    assert not got["dH"][dev(~ok)].any()
    return w


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,D,V,chunk", [(1, 8, 2, 0), (2, 24, 3, 0), (5, 64, 33, 0), (64, 64, 257, 256), (65, 72, 1000, 256),
                                         (130, 512, 2000, 512), (257, 128, 3001, 0), (300, 2048, 700, 0), (40, 2056, 1500, 512),
                                         (300, 128, 8931, 0), (513, 256, 520, 256)])
@pytest.mark.parametrize("bias", [False, True])
def test_policy_loss(dtype, M, D, V, chunk, bias):
    say("policy_loss", dtype, M, D, V, chunk, bias)
    clip, kl = (0.2, 0.3), 0.07
    c = policy_case(M + V, M, D, V, dtype, bias)
    got = policy_call(c, dtype, clip, kl, chunk=chunk, want_db=True)
    check_policy(c, dtype, clip, kl, got, db=True)
    again = policy_call(c, dtype, clip, kl, chunk=chunk)
    import torch
    assert all(torch.equal(got[k], again[k]) for k in ("loss", "losses", "logp", "dH", "dW")) and again["db"] is None
    alone = policy_call(c, dtype, clip, kl, chunk=chunk, want_dH=False)
    assert alone["dH"] is None and torch.equal(alone["dW"], got["dW"])
    none = policy_call(c, dtype, clip, kl, want_dH=False, want_dW=False)
    assert torch.equal(none["losses"], got["losses"]) and torch.equal(none["loss"], got["loss"])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_policy_loss_of_nearly_certain_tokens(dtype):
    """Where p is near one, g (1 - p) is smaller than the rounding of g p."""
    say("policy_loss certain", dtype)
    c = policy_case(5, 200, 64, 300, dtype, sure=0.5)
    ok = (c["tokens"] >= 0) & (c["tokens"] < 300)
    c["H"][ok] += 6 * c["W"][c["tokens"][ok]]
    c["H"] = host(dev(c["H"].astype(np.float32), dtype))
    z = c["H"] @ c["W"].T
    lp = z[np.arange(200), np.where(ok, c["tokens"], 0)] - np.log(np.exp(z).sum(1))
    c["old"], c["ref"] = (lp - 0.05).astype(np.float32), (lp + 0.1).astype(np.float32)
    w = check_policy(c, dtype, (0.2, 0.2), 0.05, policy_call(c, dtype, (0.2, 0.2), 0.05))
    assert np.median(w["p"][np.nonzero(ok)[0], c["tokens"][ok]]) > 0.95  # (the inputs are what they are meant to be)


@pytest.mark.parametrize("M,D,V,chunk,bias", [(1, 64, 300, 0, True), (1, 8, 2, 0, False), (3, 72, 700, 256, True),
                                              (40, 64, 100, 0, True), (40, 200, 1000, 512, False), (331, 512, 5000, 0, True)])
def test_policy_loss_of_few_tokens_a_class(M, D, V, chunk, bias):
    """In bf16 what the rounding of a token's own entry of dZ takes off is made good in all three gradients: of few
    rows one such rounding may be most of the error."""
    say("policy_loss few tokens a class", M, D, V, chunk, bias)
    c = policy_case(3 * M + V, M, D, V, "bf16", bias)
    if M < 4:  # (all of them count)
        c["tokens"] = np.abs(c["tokens"]) % V
    live = c["tokens"][(c["tokens"] >= 0) & (c["tokens"] < V)]
    assert len(live) and np.bincount(live).max() <= 16
    got = policy_call(c, "bf16", (0.2, 0.3), 0.07, chunk=chunk, want_db=True)
    check_policy(c, "bf16", (0.2, 0.3), 0.07, got, db=True, own_rounded=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift", [-300.0, 250.0])
@pytest.mark.parametrize("V", [301, 304])
def test_policy_loss_of_logits_far_from_zero(dtype, shift, V):
    """A bias that all classes share changes nothing, also where exp(-lambda) is infinite or zero and the last
    class ends inside a piece of 16 bytes."""
    say("policy_loss far from zero", dtype, shift, V)
    c = policy_case(V, 60, 64, V, dtype, True)
    c["bias"] = (c["bias"] + np.float32(shift)).astype(np.float32)
    got = policy_call(c, dtype, (0.2, 0.3), 0.07, want_db=True)
    check_policy(c, dtype, (0.2, 0.3), 0.07, got, db=True)


@pytest.mark.parametrize("M,V,classes", [(700, 300, 1), (900, 300, 2), (700, 600, 30), (1500, 130, 130), (2100, 256, 64)])
def test_policy_loss_of_many_tokens_a_class(M, V, classes):
    """More tokens of a class than are made good one by one, and more than a wavefront goes through."""
    say("policy_loss many tokens a class", M, V, classes)
    c = policy_case(M + classes, M, 64, V, "bf16", True)
    ids = np.random.default_rng(classes).permutation(V)[:classes]
    c.update(tokens=ids[np.arange(M) % classes], old=None, ref=None)
    got = policy_call(c, "bf16", (0.2, 0.3), 0.0, want_db=True, chunk=256)
    check_policy(c, "bf16", (0.2, 0.3), 0.0, got, db=True)
    again = policy_call(c, "bf16", (0.2, 0.3), 0.0, want_db=True, chunk=256)
    import torch
    assert all(torch.equal(got[k], again[k]) for k in ("dH", "dW", "db"))


@pytest.mark.parametrize("drop", ["old", "ref", "w", "old ref w", "clip"])
def test_policy_loss_without(drop):
    """No old policy (a ratio of one), no reference, unit weights, no clip."""
    say("policy_loss without", drop)
    c = policy_case(8, 100, 64, 400, "f32")
    clip = (0.2, 0.3)
    for k in drop.split():
        if k == "clip":
            clip = None
        else:
            c[k] = None
    kl = 0.0 if c["ref"] is None else 0.1
    got = policy_call(c, "f32", clip, kl)
    check_policy(c, "f32", clip or (math.inf, math.inf), kl, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_policy_loss_of_rows_that_are_not_finite(dtype):
    """Infinities and NaN in rows that are left out change nothing; in counted rows they take that row out
    alone.  (float32 tiles with such values are taken on other instructions, which round otherwise: there the
    others are checked against the reference instead of to the bit.)"""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("policy_loss nonfinite", dtype)
    M, D, V = 150, 64, 700
    c = policy_case(9, M, D, V, dtype)
    c["tokens"] = np.abs(c["tokens"]) % V
    args = lambda H, t, adv, old: pc.policy_loss(H, W, t, adv, old, clip=(0.2, 0.3))  # noqa: E731
    H, W = dev(c["H"].astype(np.float32), dtype), dev(c["W"].astype(np.float32), dtype)
    t, adv, old = torch.from_numpy(c["tokens"]).cuda(), dev(c["adv"]), dev(c["old"])
    bad = [3, 64, 65, 100, 149]
    t0 = t.clone()
    t0[bad] = -1
    want = args(H, t0, adv, old)
    H2 = H.clone()
    H2[3], H2[64, 5], H2[65] = math.nan, math.inf, -math.inf
    adv2, old2 = adv.clone(), old.clone()
    adv2[100], old2[149] = math.nan, math.nan
    c0 = dict(c, tokens=t0.cpu().numpy(), ref=None, w=None)
    for tokens, code in ((t0, pc.TOKEN_LEFT_OUT), (t, pc.TOKEN_NONFINITE)):
        got = args(H2, tokens, adv2, old2)
        status = np.zeros(M, np.int32)
        status[bad] = code
        check_policy(c0, dtype, (0.2, 0.3), 0.0, got, status=status)
        # (counted rows take a place in dW's sums, so that the others are added in other groups)
        same = ("loss", "losses", "dH") + (("dW",) if code == pc.TOKEN_LEFT_OUT else ())
        for k in same if dtype == "bf16" else ():
            assert torch.equal(got[k], want[k]), k
    # a ratio beyond every bound: clipped where that lowers the objective, left out where it does not
    adv3, old3 = torch.ones_like(adv), old.clone()
    old3[7] = old3[8] = -1e30
    adv3[8] = -1
    got = args(H, t, adv3, old3)
    assert got["status"][7] == 0 and got["losses"][7] == -np.float32(1 + np.float64(np.float32(0.3))) and not got["dH"][7].any()
    assert got["status"][8] == pc.TOKEN_NONFINITE and got["losses"][8] == 0 and torch.isfinite(got["dW"].float()).all()


@pytest.mark.parametrize("M,counted", [(1, 0), (300, 0), (300, 1), (700, 255), (700, 256), (700, 257), (700, 513), (40_000, 300),
                                       (33_000, 32_999)])
@pytest.mark.parametrize("bias", [False, True])
def test_policy_loss_of_few_counted_rows(M, counted, bias):
    """Any share of the rows left out, in blocks and scattered."""
    say("policy_loss few counted", M, counted, bias)
    D, V = 128, 300
    c = policy_case(M + counted, M, D, V, "bf16", bias)
    r = np.random.default_rng(M + counted)
    rows = np.sort(r.choice(M, counted, replace=False)) if counted % 2 else np.arange(M - counted, M)
    t = np.full(M, -1)
    t[rows] = np.abs(c["tokens"][rows]) % V
    c.update(tokens=t, old=None)
    got = policy_call(c, "bf16", (0.2, 0.3), 0.1, want_db=True, chunk=256)
    check_policy(c, "bf16", (0.2, 0.3), 0.1, got, db=True)
    assert counted or not any(got[k].any() for k in ("dH", "dW", "db", "loss"))


def test_policy_loss_without_rows_and_in_a_graph():
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("policy_loss graph")
    W = torch.randn(300, 64, device="cuda").bfloat16()
    z = torch.zeros(0, device="cuda")
    r = pc.policy_loss(W[:0], W, z.int(), z, want_db=True)
    assert r["loss"].item() == 0 and not r["dW"].any() and not r["db"].any() and r["dH"].shape == (0, 64)
    H = torch.randn(100, 64, device="cuda").bfloat16()
    t, adv = torch.randint(-1, 300, (100,), device="cuda", dtype=torch.int32), torch.randn(100, device="cuda")
    call = lambda: pc.policy_loss(H, W, t, adv, want_db=True, chunk=256)  # noqa: E731
    call()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r = call()
    for i in range(4):
        H.normal_()
        t.copy_(torch.randint(-1, 300, (100,), device="cuda"))
        g.replay()
        e = call()
        torch.cuda.synchronize()
        for k in e:
            assert torch.equal(r[k], e[k]), (i, k)


# ---- gated block ---------------------------------------------------------------------------

def ffn_case(seed, M, D, F_, O, dtype):
    r = np.random.default_rng(seed)
    c = {"x": r.normal(size=(M, D)), "wg": r.normal(size=(F_, D)) / math.sqrt(D), "wu": r.normal(size=(F_, D)) / math.sqrt(D),
         "wd": r.normal(size=(O, F_)) / math.sqrt(F_), "dy": r.normal(size=(M, O)) * 0.1}
    return {k: dev(v.astype(np.float32), dtype) for k, v in c.items()}


def product_error(A, B, eA, eB, extra=0):
    """Of A B^T with errors eA, eB in its operands: first order, the product of both, and a rounding of float per
    term of the sum (there are at most one per 16 terms and six parts; see check_policy) and `extra` more."""
    aA, aB = np.abs(A), np.abs(B)
    n = A.shape[1] + 8 + extra
    return eA @ aB.T + aA @ eB.T + eA @ eB.T + n * F * ((aA + eA) @ (aB + eB).T)


def check_ffn(c, act, dtype, got, grads=None, two_parts=False):
    """Bounds carried through the block.  a, b: their products' errors.  The
    activation's slope is at most 1.13 (and its derivative's at most 0.8), and it is itself computed to
    within 2^-20 of its argument (exponential, error function and division of a few units in the last place
    each).  Products of two factors: each one's error times the other.  two_parts: h is carried on in two parts, off by
    a rounding of what a rounding left."""
    x, wg, wu, wd = (host(c[k]) for k in ("x", "wg", "wu", "wd"))
    e = E[dtype]
    dy = host(c["dy"])
    w = ref.gated_ffn(x, wg, wu, wd, act, dy)
    z = lambda v: np.zeros_like(v)  # noqa: E731
    raw_a, raw_b = product_error(x, wg, z(x), z(wg)), product_error(x, wu, z(x), z(wu))
    f, df = ref._act(w["gate"], act)
    small = 2.0 ** -20

    def h_error(ea, eb, e):
        ef = 1.13 * ea + small * np.abs(w["gate"])
        return (ef * np.abs(w["up"]) + np.abs(f) * eb + ef * eb) * (1 + e) + (e + 2 * F) * np.abs(w["h"]) + 1e-37, ef

    eh, ef = h_error(raw_a, raw_b, e)
    ey = h_error(raw_a, raw_b, e * e)[0] if two_parts else eh
    within(got["y"], w["y"], product_error(w["h"], wd, ey, z(wd)) * (1 + e) + e * np.abs(w["y"]) + 1e-37, "y")
    ea, eb = raw_a, raw_b
    if got["gate"] is not None:
        within(got["gate"], w["gate"], ea, "gate")
        within(got["up"], w["up"], eb, "up")
    if grads is None:
        return
    edf = 0.8 * ea + small * (1 + np.abs(w["gate"]))
    edh = product_error(dy, wd.T, z(dy), z(wd.T))
    up, dh = np.abs(w["up"]), np.abs(w["dh"])
    eda = ((dh + edh) * (up + eb) * (np.abs(df) + edf) - dh * up * np.abs(df)) * (1 + e) + (e + 3 * F) * np.abs(w["da"]) + 1e-37
    edb = ((dh + edh) * (np.abs(f) + ef) - dh * np.abs(f)) * (1 + e) + (e + 2 * F) * np.abs(w["db"]) + 1e-37
    tol = {"dx": product_error(w["da"], wg.T, eda, z(wg.T), w["db"].shape[1]) + product_error(w["db"], wu.T, edb, z(wu.T), w["da"].shape[1]),
           "dw_gate": product_error(w["da"].T, x.T, eda.T, z(x.T)), "dw_up": product_error(w["db"].T, x.T, edb.T, z(x.T)),
           "dw_down": product_error(dy.T, w["h"].T, z(dy.T), eh.T)}
    for k, t in tol.items():
        within(grads[k], w[k], t * (1 + e) + e * np.abs(w[k]) + 1e-37, k)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,D,F_,O", [(1, 8, 8, 8), (1, 264, 520, 72), (2, 64, 128, 64), (3, 16, 24, 40), (7, 512, 136, 8), (8, 40, 1032, 264),
                                      (16, 256, 512, 256), (17, 1032, 264, 520), (31, 72, 200, 72), (33, 512, 384, 136), (64, 128, 264, 512),
                                      (65, 264, 136, 520), (128, 136, 648, 264), (129, 8, 264, 8), (200, 392, 72, 392), (257, 512, 776, 264),
                                      (300, 264, 1288, 520), (520, 72, 136, 1032)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_ffn(dtype, M, D, F_, O, act):
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("gated_ffn", dtype, M, D, F_, O, act)
    c = ffn_case(M + D, M, D, F_, O, dtype)
    got = pc.gated_ffn(c["x"], c["wg"], c["wu"], c["wd"], act, keep=True)
    back = lambda **kw: pc.gated_ffn_backward(c["dy"], c["x"], got["gate"], got["up"], c["wg"], c["wu"], c["wd"], act, **kw)  # noqa: E731
    grads = back()
    check_ffn(c, act, dtype, got, grads)
    plain = pc.gated_ffn(c["x"], c["wg"], c["wu"], c["wd"], act)
    assert plain["gate"] is None and torch.equal(plain["y"], got["y"])
    again = back()
    assert all(torch.equal(grads[k], again[k]) for k in grads)
    dx, dw = back(want_dw=False), back(want_dx=False)
    assert torch.equal(dx["dx"], grads["dx"]) and dx["dw_gate"] is None and dw["dx"] is None
    assert all(torch.equal(dw[k], grads[k]) for k in ("dw_gate", "dw_up", "dw_down"))


@pytest.mark.parametrize("M,D,F_,O", [(1, 8, 8, 8), (1, 336, 208, 336), (2, 336, 208, 72), (5, 64, 1032, 264), (7, 520, 64, 1032),
                                      (8, 1024, 2056, 512), (8, 72, 264, 8)])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_ffn_of_few_rows(M, D, F_, O, act):
    """Up to 8 rows in bf16 y is off by its own rounding: h is not rounded to one bf16."""
    from paper_2609_33645_amd import prunedctc as pc
    say("gated_ffn few rows", M, D, F_, O, act)
    c = ffn_case(2 * M + D, M, D, F_, O, "bf16")
    check_ffn(c, act, "bf16", pc.gated_ffn(c["x"], c["wg"], c["wu"], c["wd"], act), two_parts=True)


def test_gated_ffn_without_rows_and_of_shapes():
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("gated_ffn shapes")
    x, w, wd = torch.randn(6, 16, device="cuda"), torch.randn(24, 16, device="cuda"), torch.randn(8, 24, device="cuda")
    r = pc.gated_ffn(x[:0], w, w, wd, keep=True)
    assert r["y"].shape == (0, 8) and r["gate"].shape == (0, 24)
    g = pc.gated_ffn_backward(r["y"], x[:0], r["gate"], r["up"], w, w, wd)
    assert g["dx"].shape == (0, 16) and not any(g[k].any() for k in ("dw_gate", "dw_up", "dw_down"))
    whole = pc.gated_ffn(x, w, w, wd, keep=True)
    shaped = pc.gated_ffn(x.view(2, 3, 16), w, w, wd, keep=True)
    assert shaped["y"].shape == (2, 3, 8) and torch.equal(shaped["y"].view(6, 8), whole["y"])
    assert torch.equal(shaped["gate"].view(6, 24), whole["gate"])
    out = torch.full((6, 8), 7.0, device="cuda")
    assert pc.gated_ffn(x.T.contiguous().T, w, w.T.contiguous().T, wd, out=out)["y"] is out and torch.equal(out, whole["y"])
    for bad in (lambda: pc.gated_ffn(x[:, :15], w[:, :15], w[:, :15], wd), lambda: pc.gated_ffn(x, w, w[:16], wd),
                lambda: pc.gated_ffn(x, w, w, wd.bfloat16()), lambda: pc.gated_ffn(x, w, w, wd, out=x),
                lambda: pc.gated_ffn_backward(x, x, whole["gate"], whole["up"], w, w, wd)):
        with pytest.raises(pc.PrunedCTCError):
            bad()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [5, 300])
def test_gated_ffn_rows_do_not_meet(dtype, M):
    """Infinities and NaN in one row of x stay in that row; values that drive the activation to its ends."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("gated_ffn nonfinite", dtype, M)
    c = ffn_case(9, M, 64, 136, 72, dtype)
    for act in ("silu", "gelu"):
        want = pc.gated_ffn(c["x"], c["wg"], c["wu"], c["wd"], act)["y"]
        x = c["x"].clone()
        x[1], x[3] = math.nan, math.inf
        got = pc.gated_ffn(x, c["wg"], c["wu"], c["wd"], act)["y"]
        assert torch.isnan(got[1]).all() and not torch.isfinite(got[3]).all()
        rest = [i for i in range(M) if i not in (1, 3)]
        # (float tiles with such values are taken on other instructions)
        assert torch.equal(got[rest], want[rest]) if dtype == "bf16" else torch.allclose(got[rest], want[rest], rtol=1e-5, atol=1e-5)
        # act(-1e4) is zero, act(1e4) its argument
        big = torch.full_like(c["x"][:2], 0.0)
        big[0, 0], big[1, 0] = 1e4, -1e4
        g = torch.zeros_like(c["wg"])
        g[:, 0] = 1
        u = torch.zeros_like(g)
        u[:, 0] = 1e-4
        r = pc.gated_ffn(big, g, u, torch.eye(136, device="cuda", dtype=x.dtype)[:72].contiguous(), act, keep=True)
        assert torch.allclose(r["y"][0].float(), torch.tensor(1e4, device="cuda"), rtol=2e-2) and not r["y"][1].any()
        d = pc.gated_ffn_backward(torch.ones_like(r["y"]), big, r["gate"], r["up"], g, u,
                                  torch.eye(136, device="cuda", dtype=x.dtype)[:72].contiguous(), act)
        assert all(torch.isfinite(v.float()).all() for v in d.values())


# ---- together ------------------------------------------------------------------------------

def test_layers_in_autograd_against_the_formulas():
    """tokens -> embedding -> dropout -> gated block with residual dropout -> head -> policy loss, the head tied to
    the embedding: every gradient against the same chain in float64 (masks from the reference generator)."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("layers together")
    torch.manual_seed(3)
    V, D, F_, M, p = 211, 64, 136, 90, 0.2
    E0, wg, wu, wd = (torch.randn(s, device="cuda") / s[1] ** 0.5 for s in ((V, D), (F_, D), (F_, D), (D, F_)))
    leaves = [t.clone().requires_grad_() for t in (E0, wg, wu, wd)]
    t = torch.randint(-1, V, (M,), device="cuda", dtype=torch.int32)
    nxt, adv = torch.randint(-1, V, (M,), device="cuda"), torch.randn(M, device="cuda")
    n = M * D
    e = pc.embedding_layer(leaves[0], t, 2.0)
    x = pc.dropout_layer(e, p, 77, 0)
    y = pc.dropout_layer(pc.gated_ffn_layer(x, *leaves[1:], "gelu"), p, 77, n // 8, residual=x)
    y.retain_grad()
    out = pc.policy_loss(y.detach(), E0, nxt, adv)
    grads = list(torch.autograd.grad(y, leaves, out["dH"], retain_graph=True))
    # tied: the head's gradient and the embedding's in one buffer
    de = torch.autograd.grad(y, e, out["dH"])[0]
    tied = pc.embedding_backward(de, t, V, 2.0, out=out["dW"].clone(), accumulate=True)
    k1, k2 = (dev(ref.kept(n, p, 77, o)).view(M, D) for o in (0, n // 8))
    s = 65536 / ref.threshold(p)
    L = [q.double().requires_grad_() for q in (E0, wg, wu, wd, E0)]
    ok = (t >= 0)[:, None]
    x = torch.where(k1, torch.where(ok, L[0][t.clamp(min=0).long()], 0.0) * 2.0 * s, 0.0)
    a = x @ L[1].T
    h = 0.5 * a * (1 + torch.erf(a / math.sqrt(2))) * (x @ L[2].T)
    y64 = x + torch.where(k2, (h @ L[3].T) * s, 0.0)
    lp = torch.log_softmax(y64 @ L[4].T, 1).gather(1, nxt.clamp(min=0)[:, None])[:, 0]
    loss = -(torch.where(nxt >= 0, lp, 0.0) * adv).sum()  # (the gradient of r A at r = 1)
    want = torch.autograd.grad(loss, L)
    # float chains of a few hundred products of values of order one, against the largest of each gradient: 2e-5
    for name, g, w in (*zip(("table", "gate", "up", "down"), grads, want), ("head", out["dW"], want[4]),
                       ("tied", tied, want[0] + want[4])):
        assert float((g.double() - w).abs().max()) <= 2e-5 * float(w.abs().max()), name


def test_layers_only_form_what_is_asked():
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("layers asked")
    x, w, wd = torch.randn(5, 16, device="cuda"), torch.randn(24, 16, device="cuda"), torch.randn(16, 24, device="cuda")
    w2 = w.clone().requires_grad_()
    y = pc.gated_ffn_layer(x, w, w2, wd)
    (g,) = torch.autograd.grad(y.sum(), [w2])
    full = pc.gated_ffn(x, w, w, wd, keep=True)
    assert torch.equal(g, pc.gated_ffn_backward(torch.ones_like(x), x, full["gate"], full["up"], w, w, wd)["dw_up"])
    # the mask of the backward is the forward's, wherever the caller's counter has gone
    c = torch.tensor([5], device="cuda")
    x.requires_grad_()
    r = torch.randn(5, 16, device="cuda", requires_grad=True)
    y = pc.dropout_layer(x, 0.5, 3, c, r)
    c += 1000
    gx, gr = torch.autograd.grad(y.sum(), [x, r])
    assert torch.equal(gx, pc.dropout(torch.ones_like(x), 0.5, 3, 5)) and torch.equal(gr, torch.ones_like(r))


@pytest.mark.parametrize("op", ["dropout", "embedding", "embedding_backward", "gated_ffn", "gated_ffn_backward", "policy_loss"])
def test_on_a_given_stream_and_in_a_graph(op):
    """The same bits on another stream (its inputs let go of at once) and from a captured graph replayed with eager
    calls, other inputs and synchronizations between."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("streams and graphs", op)
    torch.manual_seed(len(op))
    M, D, F_, V = 200, 72, 136, 500
    bf = torch.bfloat16
    x, dy = (torch.randn(M, D, device="cuda").to(bf) for _ in range(2))
    wg, wu = (torch.randn(F_, D, device="cuda").to(bf) for _ in range(2))
    wd, W = torch.randn(D, F_, device="cuda").to(bf), torch.randn(V, D, device="cuda").to(bf)
    t = torch.randint(-1, V, (M,), device="cuda", dtype=torch.int32)
    adv = torch.randn(M, device="cuda")
    a, b = (torch.randn(M, F_, device="cuda") for _ in range(2))
    calls = {
        "dropout": lambda x, **k: [pc.dropout(x, 0.3, 4, 9, residual=dy, **k)],
        "embedding": lambda x, **k: [pc.embedding(x, t, 0.5, **k)],
        "embedding_backward": lambda x, **k: [pc.embedding_backward(x, t, V, dtype=torch.float32, **k)],
        "gated_ffn": lambda x, **k: list(pc.gated_ffn(x, wg, wu, wd, keep=True, **k).values()),
        "gated_ffn_backward": lambda x, **k: list(pc.gated_ffn_backward(dy, x, a, b, wg, wu, wd, **k).values()),
        "policy_loss": lambda x, **k: [v for v in pc.policy_loss(x, W, t, adv, **k).values() if v is not None],
    }
    call = calls[op]
    want = call(x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    given = [call(x, stream=s) for _ in range(3)]
    torch.cuda.current_stream().wait_stream(s)
    for got in given:
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    # an input that the caller lets go of while the call's stream still has work before it
    tmp = x.clone()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        torch.cuda._sleep(20_000_000)
    got = call(tmp, stream=s)
    del tmp
    junk = [torch.full_like(x, 9.0) for _ in range(8)]
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(g, w) for g, w in zip(got, want))
    del junk
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(x)
    for i in range(4):
        x.normal_()
        t.copy_(torch.randint(-1, V, (M,), device="cuda"))
        graph.replay()
        want = call(x)
        assert all(torch.equal(g, w) for g, w in zip(got, want)), i
        torch.cuda.synchronize()


def test_two_graphs_and_two_streams_at_once():
    """Calls in flight on two streams, and two captured graphs replayed on them, do not share memory."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("two at once")
    torch.manual_seed(1)
    V, D, F_ = 3000, 128, 264
    W = torch.randn(V, D, device="cuda").bfloat16()
    w = [torch.randn(s, device="cuda").bfloat16() for s in ((F_, D), (F_, D), (D, F_))]

    def step(x, t, adv):
        y = pc.gated_ffn(x, *w, keep=True)
        r = pc.policy_loss(y["y"], W, t, adv)
        g = pc.gated_ffn_backward(r["dH"], x, y["gate"], y["up"], *w)
        return [r["dW"], r["losses"], *g.values(), pc.embedding_backward(g["dx"], t, V)]

    data = [(torch.randn(M, D, device="cuda").bfloat16(), torch.randint(-1, V, (M,), device="cuda", dtype=torch.int32),
             torch.randn(M, device="cuda")) for M in (300, 900)]
    want = [step(*d) for d in data]
    streams = [torch.cuda.Stream() for _ in data]
    graphs, outs = [], []
    for d, s in zip(data, streams):
        s.wait_stream(torch.cuda.current_stream())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append(step(*d))
        graphs.append(g)
    for _ in range(3):
        eager = []
        for d, s, g in zip(data, streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
                eager.append(step(*d))
        torch.cuda.synchronize()
        for o, e, want_d in zip(outs, eager, want):
            assert all(torch.equal(x, z) and torch.equal(y, z) for x, y, z in zip(o, e, want_d))


def test_example_with_a_block_and_rewards():
    """Runs, with finite losses and gradients; the streams still agree with the whole utterances."""
    from paper_2609_33645_amd import fit_and_decode
    say("example")
    r = fit_and_decode.run(steps=12, beams=4, classes=60, N=3, block=72, policy=3)
    for k in ("loss_first", "loss_last", "norm_max", "reward_first", "reward_last", "policy_norm_max"):
        assert math.isfinite(r[k]), k
    assert r["norm_max"] > 0 and r["policy_norm_max"] > 0
    assert r["streams equal"] and r["predictor off by"] < 1e-3
