"""Readout with beams on the GPU, against the 64-bit references of readout_ref (all through the
public binding).

Tolerances.  A logit is a sum of D products; bf16 products are exact in float, fp32 ones round once,
and any order of D float additions errs by at most (D + 2) 2^-24 sum |h w| (to first order), which
bounds both the matrix cores' sums and the plain ones.  A log probability adds the normaliser's error
(the largest of its logits' errors, and 2e-5 for its float partial sums, the bar of the normaliser's own
tests) and one rounding.  A search step makes at most eight roundings of values below 64 in magnitude
relative to the best prefix, plus 4e-7 for each of its mass additions: 3.2e-5 a frame at the very most,
and one rounding of the score at the end."""
import math

import numpy as np
import pytest

from tests import readout_ref as ref
from tests.gpu_util import say

pytestmark = pytest.mark.gpu

STEP = 3.2e-5


def bf16_round(x):
    from paper_2609_33645_amd import workloads
    return workloads.round_to_bf16(np.asarray(x, np.float32))


def head(seed, M, D, V, dtype, scale=1.0):
    r = np.random.default_rng(seed)
    H = (r.normal(size=(M, D)) * scale).astype(np.float32)
    W = (r.normal(size=(V, D)) / math.sqrt(D)).astype(np.float32)
    return (bf16_round(H), bf16_round(W)) if dtype == "bf16" else (H, W)


def dev(x, dtype=None):
    import torch
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t.to({"bf16": torch.bfloat16, "f32": torch.float32}[dtype]) if dtype else t


def check_candidates(H, W, C, blank, bias, dtype, got):
    z = ref.logits(H, W, bias)
    M, V = z.shape
    mass = np.abs(H.astype(np.float64)) @ np.abs(W.astype(np.float64)).T + (0 if bias is None else np.abs(
        np.where(np.isfinite(bias), bias, 0.0)))
    err = (H.shape[1] + 2) * 2.0 ** -24 * mass
    ids, logp, bl = (got[k].cpu().numpy() for k in ("ids", "logp", "blank_logp"))
    assert ids.shape == logp.shape == (M, C) and bl.shape == (M,)
    top = z.max(1)
    lam = top + np.log(np.exp(z - top[:, None]).sum(1))
    rbl = z[:, blank] - lam
    tol_lam = err.max(1) + 2e-5
    zz = z.copy()
    zz[:, blank] = -np.inf
    k = np.minimum(C, (zz > -np.inf).sum(1))  # classes that exist
    for m in range(M):
        n = k[m]
        assert (ids[m, n:] == -1).all() and np.isneginf(logp[m, n:]).all(), (m, ids[m], n)
        own = ids[m, :n]
        assert len(set(own.tolist())) == n and (own != blank).all() and (own >= 0).all() and (own < V).all(), (m, own)
        d = np.abs(logp[m, :n] - (z[m, own] - lam[m]))
        assert (d <= err[m, own] + tol_lam[m] + 2.0 ** -23 * np.abs(logp[m, :n])).all(), (m, d.max())
        assert (np.diff(logp[m, :n]) <= 0).all()
        # nothing left out stands above what was taken by more than both errors
        rest = zz[m].copy()
        rest[own] = -np.inf
        if n == C and np.isfinite(rest.max()):
            worst = own[np.argmin(z[m, own])]
            e = err[m].max()
            assert rest.max() - z[m, worst] <= 2 * e, (m, rest.max(), z[m, worst], e)
    fin = np.isfinite(rbl)
    assert (np.abs(bl[fin] - rbl[fin]) <= (err[:, blank] + tol_lam + 2.0 ** -23 * np.abs(bl))[fin]).all()
    assert np.isneginf(bl[~fin]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,D,V,C,blank", [
    (1, 8, 2, 1, 0), (1, 8, 2, 4, 1), (3, 24, 3, 64, 2), (5, 64, 33, 8, 32), (64, 64, 257, 64, 0), (65, 72, 1000, 16, 7),
    (130, 512, 5000, 16, 4999), (257, 128, 8931, 33, 0), (7, 4096, 3001, 8, 0), (300, 2048, 700, 5, 3), (40, 512, 70_001, 16, 0)])
@pytest.mark.parametrize("bias", [False, True])
def test_candidates(dtype, M, D, V, C, blank, bias):
    from paper_2609_33645_amd import prunedctc as pc
    say("candidates", dtype, M, D, V, C, blank, bias)
    H, W = head(M + V, M, D, V, dtype, 3.0)
    b = (np.random.default_rng(V).normal(size=V) * 2).astype(np.float32) if bias else None
    got = pc.frame_candidates(dev(H, dtype), dev(W, dtype), C, blank, None if b is None else dev(b))
    check_candidates(H, W, C, blank, b, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,D,V,C,blank", [
    (70, 8, 700, 3, 1), (513, 24, 5003, 16, 4999), (600, 64, 9001, 5, 0), (512, 128, 40_000, 64, 0),  # formed again
    (513, 128, 1501, 9, 3), (700, 1032, 259, 64, 258)])                                               # kept
def test_candidates_either_way(dtype, M, D, V, C, blank):
    """Logits formed again and kept, for few frames and many."""
    from paper_2609_33645_amd import prunedctc as pc
    say("either way", dtype, M, D, V, C, blank)
    H, W = head(M * V, M, D, V, dtype, 3.0)
    b = np.random.default_rng(V).normal(size=V).astype(np.float32)
    got = pc.frame_candidates(dev(H, dtype), dev(W, dtype), C, blank, dev(b))
    check_candidates(H, W, C, blank, b, dtype, got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["zero", "few", "steps"])
def test_candidates_ties(dtype, kind):
    """Equal logits (exact sums of small whole numbers): the lowest classes first, also where more
    blocks are equal than the ordering's list holds."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    say("ties", dtype, kind)
    M, D, V, C, blank = 5, 32, 20_000, 20, 4
    r = np.random.default_rng(3)
    H = np.ones((M, D), np.float32)
    W = np.zeros((V, D), np.float32)
    if kind == "few":
        W[:, 0] = r.integers(0, 3, size=V)
    elif kind == "steps":
        W[:, 0] = np.arange(V) // 9000  # 344 equal blocks on top, 281 and more below
        W[9001, 1] = 7
    got = pc.frame_candidates(dev(H, dtype), dev(W, dtype), C, blank)
    ids, _, _ = ref.candidates(ref.logits(H, W), C, blank)
    assert np.array_equal(got["ids"].cpu().numpy(), ids)
    again = pc.frame_candidates(dev(H, dtype), dev(W, dtype), C, blank)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("open_classes", [0, 1, 9, 40])
def test_candidates_masked_vocabulary(dtype, open_classes):
    """A bias of -inf, or the type's lowest value, on all but a few classes."""
    from paper_2609_33645_amd import prunedctc as pc
    say("masked", dtype, open_classes)
    M, D, V, C, blank = 9, 64, 3000, 16, 11
    H, W = head(5, M, D, V, dtype)
    r = np.random.default_rng(open_classes)
    for low in (-np.inf, np.finfo(np.float32).min):
        b = np.full(V, low, np.float32)
        b[blank] = 0.5
        b[r.choice(np.setdiff1d(np.arange(V), [blank]), open_classes, replace=False)] = 0.25
        got = pc.frame_candidates(dev(H, dtype), dev(W, dtype), C, blank, dev(b))
        if np.isinf(low):
            check_candidates(H, W, C, blank, b, dtype, got)
        else:
            n = min(C, open_classes)
            ids, logp = got["ids"].cpu().numpy(), got["logp"].cpu().numpy()
            rids, rlogp, _ = ref.candidates(ref.logits(H, W, b), C, blank)
            assert all(set(ids[m, :n]) == set(rids[m, :n]) for m in range(M))
            assert (logp[:, n:] < -1e38).all()


def test_candidates_masked_blank_and_all():
    from paper_2609_33645_amd import prunedctc as pc
    H, W = head(6, 4, 64, 500, "bf16")
    b = np.zeros(500, np.float32)
    b[3] = -np.inf
    got = pc.frame_candidates(dev(H, "bf16"), dev(W, "bf16"), 8, 3, dev(b))
    check_candidates(H, W, 8, 3, b, "bf16", got)
    got = pc.frame_candidates(dev(H, "bf16"), dev(W, "bf16"), 8, 3, dev(np.full(500, -np.inf, np.float32)))
    assert (got["ids"].cpu().numpy() == -1).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("top", [0, 700])
def test_candidates_certain_frames(dtype, top):
    """Frames of one nearly certain class, its logit near 200, where a logit's own rounding is 1e-5: the class's
    log-probability holds neither that rounding nor the loss of 5,000 classes that are each below a sum's last
    bit.  The normaliser rounds the sum of such a frame some 16 times, at 2^-24 each at most, and its terms'
    exponents at 4 x 2^-24 together."""
    from paper_2609_33645_amd import prunedctc as pc
    say("certain", dtype, top)
    M, D, V, C, blank = 70, 512, 5000, 8, 0
    r = np.random.default_rng(top)
    h = r.standard_normal(D)
    z = r.uniform(165.0, 183.0, V)
    z[top] = 200.0
    W = z[:, None] * h[None, :] / (h @ h) + 0.002 * r.standard_normal((V, D))
    H = h[None, :] * r.uniform(0.97, 1.03, M)[:, None]
    H, W = (bf16_round(x) if dtype == "bf16" else x.astype(np.float32) for x in (H, W))
    got = pc.frame_candidates(dev(H, dtype), dev(W, dtype), C, blank)
    z = H.astype(np.float64) @ W.astype(np.float64).T
    x = z - z[:, top:top + 1]
    x[:, top] = -np.inf
    want = -np.log1p(np.exp(x).sum(1))
    out = got["blank_logp"] if top == blank else got["logp"][:, 0]
    if top != blank:
        assert (got["ids"][:, 0] == top).all()
    assert np.abs(out.cpu().numpy().astype(np.float64) - want).max() <= 20 * 2.0**-24


@pytest.mark.parametrize("M,D,V,C", [
    (100, 520, 40_001, 16), (65, 4096, 33_003, 3), (128, 512, 70_001, 64),  # one tile of 128 frames
    (64, 1032, 40_001, 5), (130, 1024, 12_000, 16),                         # rows copied 64 deep
    (700, 512, 230_001, 16), (1025, 2048, 40_007, 8)])                      # frames from H transposed
@pytest.mark.parametrize("bias", [False, True])
def test_candidates_tiles(M, D, V, C, bias):
    """The product's other tiles, up to 50 frames of them against the definition."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    say("tiles", M, D, V, C, bias)
    H, W = head(M + V + D, M, D, V, "bf16", 3.0)
    b = (np.random.default_rng(V).normal(size=V) * 2).astype(np.float32) if bias else None
    got = pc.frame_candidates(dev(H, "bf16"), dev(W, "bf16"), C, 3, None if b is None else dev(b))
    rows = np.unique(np.concatenate([[0, M - 1], np.random.default_rng(M).integers(0, M, 48)]))
    at = torch.from_numpy(rows).cuda()
    check_candidates(H[rows], W, C, 3, b, "bf16", {k: v[at] for k, v in got.items()})


def test_candidates_without_frames():
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    W = torch.randn(100, 64, device="cuda")
    got = pc.frame_candidates(W[:0], W, 8)
    assert got["ids"].shape == (0, 8) and got["blank_logp"].shape == (0,)


def test_candidates_passes():
    """More frames than one pass over the vocabulary takes: each as if it were alone."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    M, D, V = 700, 64, 524_288  # a pass takes 2,048 frames
    r = torch.Generator(device="cuda")
    r.manual_seed(1)
    H = torch.randn(M, D, generator=r, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, D, generator=r, device="cuda") / 8).to(torch.bfloat16)
    big = H.repeat(8, 1)
    one, many = pc.frame_candidates(H, W, 8), pc.frame_candidates(big, W, 8)
    for k in one:
        assert torch.allclose(many[k].float(), one[k].float().repeat(*([8] + [1] * (one[k].dim() - 1))), atol=2e-5), k


def test_candidates_passes_with_logits():
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    M, D, V, C = 500, 512, 30_001, 64  # a pass takes 3,840 frames
    r = torch.Generator(device="cuda")
    r.manual_seed(2)
    H = torch.randn(M, D, generator=r, device="cuda").to(torch.bfloat16)
    W = (torch.randn(V, D, generator=r, device="cuda") / 8).to(torch.bfloat16)
    one, many = pc.frame_candidates(H, W, C), pc.frame_candidates(H.repeat(8, 1), W, C)
    assert torch.equal(many["ids"], one["ids"].repeat(8, 1))
    for k in ("logp", "blank_logp"):
        assert torch.allclose(many[k], one[k].repeat(*([8] + [1] * (one[k].dim() - 1))), atol=2e-5), k


# ---- the search ----------------------------------------------------------------------------

def random_frames(seed, T, C, V, scale=3.0):
    """Falling scores over distinct classes from a small alphabet: labels repeat, prefixes meet."""
    r = np.random.default_rng(seed)
    ids = np.stack([r.permutation(np.arange(1, V))[:C] for _ in range(T)]) if T else np.zeros((0, C), int)
    z = r.exponential(scale, size=(T, C + 1))
    z = -(z - z.min(1, keepdims=True)) if T else z
    lse = np.log(np.exp(z).sum(1, keepdims=True)) if T else z
    z = (z - lse).astype(np.float32)
    return ids.astype(np.int32), -np.sort(-z[:, 1:], 1), z[:, 0]


def clear_frames(seed, T, C, V, K, bonus, least=1e-4, tries=400):
    """Frames whose search has no decision closer than `least`."""
    for k in range(tries):
        ids, lp, bl = random_frames(seed + 7919 * k, T, C, V)
        s = ref.Search(K, bonus).run(ids, lp, bl)
        if s.gap > least:
            return ids, lp, bl, s.result()
    raise AssertionError("no clear case")


def run_search(parts, K, bonus=0.0, chunks=None, max_tokens=None, max_frames=None):
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    N, C = len(parts), parts[0][0].shape[1]
    T = [len(q[2]) for q in parts]
    b = pc.BeamSearch(N, K, max_frames or max(max(T), 1), bonus)
    for t0, t1 in chunks or [(0, max(T))]:
        cut = [(q[0][t0:t1], q[1][t0:t1], q[2][t0:t1]) for q in parts]
        cat = [dev(np.concatenate([q[i] for q in cut])) for i in range(3)]
        b.advance(*cat, [len(q[2]) for q in cut])
    assert b.frames_done.tolist() == T
    r = b.result(max_tokens)
    torch.cuda.synchronize()
    del C
    return {k: v.cpu().numpy() for k, v in r.items()}


def check_result(r, n, want, T, tol=None):
    K = r["scores"].shape[1]
    tol = T * STEP if tol is None else tol
    for k in range(K):
        if k >= len(want):
            assert r["token_lengths"][n, k] == -1 and np.isneginf(r["scores"][n, k])
            assert (r["tokens"][n, k] == -1).all()
            continue
        y, s = want[k]
        assert r["token_lengths"][n, k] == len(y), (n, k, y)
        assert r["tokens"][n, k, :len(y)].tolist() == list(y), (n, k)
        assert (r["tokens"][n, k, len(y):] == -1).all()
        assert abs(r["scores"][n, k] - s) <= tol + 2.0 ** -23 * abs(s), (n, k, r["scores"][n, k], s)


@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 8, 11, 16, 17, 32])
@pytest.mark.parametrize("C,V", [(1, 2), (2, 4), (5, 7), (16, 20), (64, 70)])
@pytest.mark.parametrize("bonus", [0.0, -0.7, 0.4])
def test_search(K, C, V, bonus):
    say("search", K, C, V, bonus)
    T = (1, 2, 7, 24)
    cases = [clear_frames(1000 * K + 10 * C + t, t, C, V, K, bonus, least=2e-5) for t in T]
    r = run_search([c[:3] for c in cases], K, bonus)
    for n, c in enumerate(cases):
        check_result(r, n, c[3], T[n])


def test_search_meets_dropped_prefixes():
    """Two classes and two beams over many frames: prefixes leave the beam and come back."""
    cases = [clear_frames(50 + i, 30, 2, 3, 2, 0.0, least=2e-5) for i in range(12)]
    r = run_search([c[:3] for c in cases], 2)
    for n, c in enumerate(cases):
        check_result(r, n, c[3], 30)


@pytest.mark.parametrize("N", [1, 255, 256, 257, 600])
def test_search_many_utterances(N):
    """Utterances in groups of a launch, some without frames; each as if it were alone."""
    say("utterances", N)
    r = np.random.default_rng(N)
    T = r.integers(0, 6, size=N)
    parts = [random_frames(10 * n + 3, int(T[n]), 3, 5) for n in range(N)]
    got = run_search(parts, 4, max_frames=6, max_tokens=6)
    for n in range(N):
        s = ref.Search(4).run(*parts[n])
        if s.gap > 2e-5:
            check_result(got, n, s.result(), int(T[n]))


@pytest.mark.parametrize("K", [3, 8, 32])
def test_search_in_pieces(K):
    """Frame by frame and in uneven pieces: bit for bit the whole run's result."""
    parts = [random_frames(s, t, 6, 9) for s, t in ((1, 40), (2, 23), (3, 1))]
    whole = run_search(parts, K)
    for chunks in ([(t, t + 1) for t in range(40)], [(0, 0), (0, 13), (13, 14), (14, 40)]):
        got = run_search(parts, K, chunks=chunks)
        assert all(np.array_equal(whole[k], got[k]) for k in whole)


def test_parents_carry_state():
    """A caller's own label lists, reordered by the parents of every call, stay the beams' prefixes."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    N, K, T, C = 3, 6, 40, 5
    parts = [random_frames(20 + n, T, C, 8) for n in range(N)]
    b = pc.BeamSearch(N, K, T)
    have = torch.zeros(N, K, T, dtype=torch.int32, device="cuda")  # labels + 1, 0 past the end
    t = 0
    for step in (1, 1, 2, 5, 1, 7, 3, 20):
        cat = [dev(np.concatenate([q[i][t:t + step] for q in parts])) for i in range(3)]
        parents = b.advance(*cat, [step] * N)
        t += step
        pc.beam_reorder([have], parents)
        now = b.result(T)
        tok = now["tokens"] + 1
        # what each beam had before the call is the beginning of what it has now
        assert ((have == 0) | (have == tok)).all()
        assert ((now["token_lengths"] - (have > 0).sum(2)) <= step).all()
        assert ((parents >= 0) == (now["token_lengths"] >= 0)).all()
        have.copy_(tok)
    assert t == T


def test_search_impossible_frames():
    """Frames that offer nothing, no numbers, or blank alone."""
    ids = np.array([[3, 5], [-1, -1], [3, -1], [4, 3]], np.int32)
    lp = np.array([[-0.1, -3.0], [-np.inf, np.nan], [np.nan, -0.5], [-1.0, -1.5]], np.float32)
    bl = np.array([-2.5, -0.25, -0.125, -0.5], np.float32)
    s = ref.Search(4)
    for t in range(4):
        s.step([v if l > -np.inf else -1 for v, l in zip(ids[t], lp[t])], lp[t], float(bl[t]))
    dead = bl.copy()
    dead[1:] = (-np.inf, np.nan, -np.inf)
    none = np.full_like(ids, -1)
    r = run_search([(ids, lp, bl), (none, lp, dead), (none, lp, bl)], 4)
    check_result(r, 0, s.result(), 4)
    check_result(r, 1, [], 4)
    check_result(r, 2, [((), float(bl.sum()))], 4)
    # no frames at all: the empty prefix
    empty = (ids[:0], lp[:0], bl[:0])
    r = run_search([empty, empty], 3, max_tokens=2)
    check_result(r, 0, [((), 0.0)], 1)


def test_long_prefix():
    """Prefixes of thousands of labels (the result's walk takes 63 segments of 32 at a time), cut to
    max_tokens."""
    T = 5000
    r = np.random.default_rng(0)
    path = r.integers(1, 1000, size=T)
    path[1:] += (path[1:] == path[:-1])
    ids = np.stack([path, path + 2000], 1).astype(np.int32)
    lp = np.tile(np.array([[-0.01, -9.0]], np.float32), (T, 1))
    lp[100, 1] = -6.0
    bl = np.full(T, -12.0, np.float32)
    got = run_search([(ids, lp, bl), (ids[:2017], lp[:2017], bl[:2017])], 2, max_frames=T)
    want = path.tolist()
    assert got["tokens"][0, 0].tolist() == want and got["token_lengths"].tolist() == [[T, T], [2017, 2017]]
    assert got["tokens"][1, 0, :2017].tolist() == want[:2017] and (got["tokens"][1, :, 2017:] == -1).all()
    second = want.copy()
    second[100] += 2000
    assert got["tokens"][0, 1].tolist() == second
    for cut in (1, 31, 32, 33, 2016):
        short = run_search([(ids, lp, bl)], 2, max_frames=T, max_tokens=cut)
        assert short["tokens"][0, 1].tolist() == second[:cut] and short["token_lengths"][0, 0] == T
    # far beyond a float's resolution of its total, the score is still the sum
    assert abs(got["scores"][0, 0] - T * float(np.float32(-0.01))) < T * 1e-6


def test_search_state_is_reset_and_bounded():
    from paper_2609_33645_amd import prunedctc as pc
    ids, lp, bl = random_frames(4, 10, 4, 6)
    b = pc.BeamSearch(1, 4, 10)
    args = (dev(ids), dev(lp), dev(bl), [10])
    b.advance(*args)
    first = b.result()
    with pytest.raises(pc.PrunedCTCError) as e:
        b.advance(dev(ids[:1]), dev(lp[:1]), dev(bl[:1]), [1])
    assert e.value.code == -3 and b.frames_done.tolist() == [10]
    b.reset()
    b.advance(*args)
    second = b.result()
    assert all(bool((first[k] == second[k]).all()) for k in first)
    for bad in ((dev(ids), dev(lp), dev(bl), [9]), (dev(ids[:, :3]), dev(lp), dev(bl), [10]),
                (dev(ids), dev(lp), dev(bl), [5, 5]), (dev(ids).cpu(), dev(lp), dev(bl), [10])):
        with pytest.raises(pc.PrunedCTCError):
            b.advance(*bad)


def test_search_strided_and_other_types():
    """Candidates as views and in other types: converted, not misread."""
    ids, lp, bl = random_frames(9, 12, 4, 6)
    want = run_search([(ids, lp, bl)], 4)
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    wide = torch.zeros(12, 8, device="cuda")
    wide[:, ::2] = dev(lp)
    b = pc.BeamSearch(1, 4, 12)
    b.advance(dev(ids).long(), wide[:, ::2], dev(bl).double(), np.array([12], np.int64))
    got = b.result()
    assert all(np.array_equal(want[k], got[k].cpu().numpy()) for k in want)


# ---- reordering ------------------------------------------------------------------------------

@pytest.mark.parametrize("K", [1, 2, 4, 7, 8, 13, 16, 31, 32])
@pytest.mark.parametrize("in_place", [False, True])
def test_reorder(K, in_place):
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    say("reorder", K, in_place)
    g = torch.Generator(device="cuda")
    g.manual_seed(K)
    N = 3
    shapes = [((1,), torch.uint8), ((3,), torch.bfloat16), ((5, 7), torch.float32), ((16,), torch.uint8), ((17,), torch.int8),
              ((2, 1024), torch.float64), ((4097,), torch.uint8), ((0,), torch.float32), ((), torch.int32),
              ((3, 1111), torch.bfloat16)]
    states = [torch.randint(-100, 100, (N, K) + s, generator=g, device="cuda").to(d) for s, d in shapes]
    parents = torch.randint(0, K, (N, K), generator=g, device="cuda", dtype=torch.int32)
    parents[0, 0], parents[1, K - 1], parents[2, K // 2] = -1, K, 2 ** 31 - 1
    src = torch.where((parents >= 0) & (parents < K), parents, torch.arange(K, device="cuda", dtype=torch.int32)).long()
    want = [torch.stack([t[n][src[n]] for n in range(N)]) for t in states]
    before = [t.clone() for t in states]
    out = None if in_place else [torch.empty_like(t) for t in states]
    got = pc.beam_reorder(states, parents, out)
    for g_, w, t, b in zip(got, want, states, before):
        assert torch.equal(g_, w)
        assert in_place or torch.equal(t, b)


def test_reorder_many_tensors_odd_addresses():
    """More tensors than a launch's table holds, at addresses of every alignment; what lies between
    them is left alone."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    N, K, n = 2, 4, 150
    sizes = [(i * 37) % 301 + 1 for i in range(n)]
    total = sum(N * K * s + 3 for s in sizes)
    r = np.random.default_rng(0)
    flat = dev(r.integers(0, 255, size=total).astype(np.uint8))
    dest = dev(np.full(total, 77, np.uint8))
    parents = dev(r.integers(0, K, size=(N, K)).astype(np.int32))
    want = torch.full_like(dest, 77)
    states, outs, at = [], [], 0
    for s in sizes:
        states.append(flat[at:at + N * K * s].view(N, K, s))
        outs.append(dest[at:at + N * K * s].view(N, K, s))
        want[at:at + N * K * s].view(N, K, s).copy_(
            torch.stack([states[-1][i][parents[i].long()] for i in range(N)]))
        at += N * K * s + 3
    pc.beam_reorder(states, parents, outs)
    assert torch.equal(dest, want)


def test_reorder_refusals():
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    p = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    ok = torch.zeros(2, 4, 5, device="cuda")
    for states, out in (([ok.cpu()], None), ([ok[:, :3]], None), ([ok.transpose(0, 1)], None), ([ok[:, :, ::2]], None),
                        ([ok], []), ([ok], [ok.half()]), ([ok], [ok[:, :, :4]])):
        with pytest.raises(pc.PrunedCTCError):
            pc.beam_reorder(states, p, out)
    with pytest.raises(pc.PrunedCTCError):
        pc.beam_reorder([ok], p.long())
    with pytest.raises(pc.PrunedCTCError):
        pc.beam_reorder([torch.zeros(2, 33, 1, device="cuda")], torch.zeros(2, 33, dtype=torch.int32, device="cuda"))
    assert pc.beam_reorder([], p) == []


# ---- frames to label sequences ---------------------------------------------------------------

def spoken(seed, T, D, V, dtype, peak=14.0):
    """A head, frames that speak random transcripts through it, one frame in six torn between two
    classes."""
    r = np.random.default_rng(seed)
    W = (r.normal(size=(V, D)) / math.sqrt(D)).astype(np.float32)
    W = bf16_round(W) if dtype == "bf16" else W
    M = int(sum(T))
    path = np.where(r.random(M) < 0.4, r.integers(0, V, size=M), 0)
    again = np.flatnonzero(r.random(M) < 0.3)[1:]
    path[again] = path[again - 1]
    H = r.normal(size=(M, D)).astype(np.float32) * 0.5 + peak * W[path]
    torn = np.flatnonzero(r.random(M) < 1 / 6)
    H[torn] += (peak - r.uniform(0.3, 4.0, size=len(torn)))[:, None].astype(np.float32) * W[r.integers(0, V, size=len(torn))]
    return (bf16_round(H), W) if dtype == "bf16" else (H.astype(np.float32), W)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,D,V,K,C,blank,bonus,bias", [
    ((1,), 64, 50, 2, 3, 0, 0.0, False), ((30, 1, 17), 64, 300, 4, 8, 0, 0.0, True), ((60, 45), 512, 5000, 8, 16, 0, -0.3, False),
    ((25,), 72, 1001, 5, 33, 1000, 0.2, True), ((40, 40, 40, 8), 2048, 900, 3, 4, 0, 0.0, False), ((12,), 64, 5, 32, 64, 2, 0.0, False)])
def test_decode(dtype, T, D, V, K, C, blank, bonus, bias):
    from paper_2609_33645_amd import prunedctc as pc
    say("decode", dtype, T, D, V, K, C)
    b = (np.random.default_rng(1).normal(size=V) * 0.3).astype(np.float32) if bias else None
    for seed in range(100, 140):
        H, W = spoken(seed, T, D, V, dtype)
        ids, lp, bl = ref.candidates(ref.logits(H, W, b), C, blank)
        off = np.concatenate([[0], np.cumsum(T)])
        runs = [ref.Search(K, bonus).run(ids[s:e], lp[s:e], bl[s:e]) for s, e in zip(off[:-1], off[1:])]
        if min(s.gap for s in runs) > 1e-5:
            break
    got = pc.beam_decode(dev(H, dtype), dev(W, dtype), list(T), K, C, blank, None if b is None else dev(b), bonus)
    check_candidates(H, W, C, blank, b, dtype, got)
    r = {k: got[k].cpu().numpy() for k in ("tokens", "token_lengths", "scores")}
    assert r["tokens"].shape == (len(T), K, max(T))
    mass = (np.abs(H.astype(np.float64)) @ np.abs(W.astype(np.float64)).T).max()
    per_frame = 2 * (D + 2) * 2.0 ** -24 * mass + 2e-5 + STEP
    for n, s in enumerate(runs):
        # the best prefix's decisions are far from ties; the others' where the search had no close one
        want = s.result()
        check_result({k: v[:, :1] for k, v in r.items()}, n, want[:1], T[n], T[n] * per_frame)
        if s.gap > 2 * per_frame:
            check_result(r, n, want, T[n], T[n] * per_frame)


def test_decode_equals_its_stages():
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    T = [33, 20, 47]
    H, W = spoken(7, T, 128, 3000, "bf16")
    Hd, Wd = dev(H, "bf16"), dev(W, "bf16")
    whole = pc.beam_decode(Hd, Wd, T, 6, 12, token_bonus=0.1)
    c = pc.frame_candidates(Hd, Wd, 12)
    b = pc.BeamSearch(3, 6, 47, 0.1)
    b.advance(c["ids"], c["logp"], c["blank_logp"], T)
    for k, v in {**c, **b.result()}.items():
        assert torch.equal(whole[k], v), k
    cut = pc.beam_decode(Hd, Wd, T, 6, 12, token_bonus=0.1, max_tokens=2)
    assert torch.equal(cut["tokens"], whole["tokens"][:, :, :2]) and torch.equal(cut["token_lengths"], whole["token_lengths"])
    with pytest.raises(pc.PrunedCTCError) as e:
        pc.beam_decode(Hd, Wd, [100, 0], 6, 12)
    assert e.value.code == -3
    with pytest.raises(pc.PrunedCTCError):
        pc.beam_decode(Hd, Wd, [100, 1], 6, 12)


def test_greedy_is_one_beam_of_certain_frames():
    """Where every frame is nearly certain, the best prefix is the greedy readout."""
    from paper_2609_33645_amd import prunedctc as pc
    T = [50, 31]
    r = np.random.default_rng(2)
    W = bf16_round(r.normal(size=(2000, 256)) / 16)
    path = np.where(r.random(81) < 0.5, r.integers(0, 2000, size=81), 0)
    H = bf16_round(r.normal(size=(81, 256)) * 0.1 + 30 * W[path])
    g = pc.greedy_decode(dev(H, "bf16"), dev(W, "bf16"), T)
    b = pc.beam_decode(dev(H, "bf16"), dev(W, "bf16"), T, 4, 8)
    for n in range(2):
        k = int(b["token_lengths"][n, 0])
        assert b["tokens"][n, 0, :k].tolist() == g["tokens"][n]


# ---- streams and graphs ------------------------------------------------------------------------

def test_other_stream():
    """Calls on another stream than the current one, the current one kept busy with the allocator's
    memory meanwhile."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    T = [80, 60]
    H, W = spoken(8, T, 256, 4000, "bf16")
    Hd, Wd = dev(H, "bf16"), dev(W, "bf16")
    want = pc.beam_decode(Hd, Wd, T, 8, 16)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(5):
        got = pc.beam_decode(Hd, Wd, T, 8, 16, stream=side)
        junk = [torch.full((1 << 18,), 7, device="cuda") for _ in range(8)]
        side.synchronize()
        assert all(torch.equal(want[k], got[k]) for k in want)
        del junk


def test_other_stream_keeps_the_callers_tensors():
    """Tensors let go of right after a call on a busy stream, their memory asked for again on the current one."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    T = [80, 60]
    H, W = spoken(8, T, 256, 4000, "bf16")
    want = pc.beam_decode(dev(H, "bf16"), dev(W, "bf16"), T, 8, 16)
    grads = [torch.randn(300_000, device="cuda") for _ in range(3)]
    norm = pc.clip_grad_norm(grads, 1.0, out=[torch.empty_like(g) for g in grads])["norm"].clone()
    a = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    for _ in range(3):
        Hd, Wd, gs = dev(H, "bf16"), dev(W, "bf16"), [g.clone() for g in grads]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(4):
                torch.mm(a, a)
        got = pc.beam_decode(Hd, Wd, T, 8, 16, stream=side)
        clipped = pc.clip_grad_norm(gs, 1.0, out=[torch.empty_like(g) for g in gs], stream=side)
        sizes = [(t.shape, t.dtype) for t in (Hd, Wd, *gs)]
        del Hd, Wd, gs
        junk = [torch.full(s, 7, dtype=d, device="cuda") for s, d in sizes]
        torch.cuda.synchronize()
        assert all(torch.equal(want[k], got[k]) for k in want)
        assert torch.equal(clipped["norm"], norm)
        del junk


def test_graph_replays():
    """A captured step (candidates, one frame of search, reordering) replayed on new frames."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    N, D, V, K, C, T = 3, 64, 700, 4, 8, 6
    H, W = spoken(9, [T] * N, D, V, "bf16", peak=8.0)
    Hd, Wd = dev(H, "bf16").view(N, T, D), dev(W, "bf16")
    frame = torch.empty(N, D, dtype=torch.bfloat16, device="cuda")
    state = torch.zeros(N, K, 16, device="cuda")

    def step(b, bits):
        c = pc.frame_candidates(frame, Wd, C)
        bits.append(pc.beam_reorder([state], b.advance(c["ids"], c["logp"], c["blank_logp"], [1] * N))[0])
        return c

    # one graph per position in the stream (the frames before are part of the capture)
    b = pc.BeamSearch(N, K, T)
    frame.copy_(Hd[:, 0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(b, [])
    torch.cuda.current_stream().wait_stream(side)
    b.reset()
    graphs = []
    for t in range(T):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(b, [])
        graphs.append(g)
    for rep in range(3):
        order = list(range(T)) if rep != 1 else list(reversed(range(T)))  # another utterance's frames
        b.reset()
        state.copy_(torch.arange(K, device="cuda").float()[None, :, None].expand(N, K, 16))
        for i, t in enumerate(order):
            frame.copy_(Hd[:, t])
            graphs[i].replay()
            torch.cuda.synchronize()
        b._done[:] = T  # the replays advanced the state, not the host's count
        got, moved = b.result(), state.clone()
        e = pc.BeamSearch(N, K, T)
        state.copy_(torch.arange(K, device="cuda").float()[None, :, None].expand(N, K, 16))
        for t in order:
            frame.copy_(Hd[:, t])
            step(e, [])
        want = e.result()
        assert all(torch.equal(got[k], want[k]) for k in want)
        assert torch.equal(moved, state)


# ---- gradient norm and clipping ------------------------------------------------------------------

def clip_inputs(seed, spec, scale=0.02):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * scale).to(torch.bfloat16 if t == "b" else torch.float32)
            for t, n in spec]


def check_clip(before, got, r, max_norm):
    """Squares and their sum in double: the norm is the exact one to a float rounding (and sums of
    double, 1e-12); the scale another; a product and its rounding to bf16 one each."""
    import torch
    exact = math.sqrt(sum(float(t.double().square().sum()) for t in before))
    s = min(1.0, max_norm / (exact + 1e-6))
    assert abs(float(r["norm"]) - exact) <= 2.0 ** -24 * 1.0001 * exact + 1e-45
    assert abs(float(r["scale"]) - s) <= 2.0 ** -24 * 1.0001 * s
    for b, o in zip(before, got):
        w = b.double() * s
        tol = (2.0 ** -8 if b.dtype == torch.bfloat16 else 2.0 ** -22.9) * w.abs() + 2.0 ** -133
        assert ((o.double() - w).abs() <= tol).all()


SPECS = {
    "one": [("f", 1)], "none": [("f", 0), ("b", 0)], "odd": [("f", 7), ("b", 1), ("f", 0), ("b", 33), ("f", 8191), ("b", 16385)],
    "chunks": [("f", 8192), ("b", 16384), ("f", 8193), ("f", 1_000_003), ("b", 2_000_001), ("f", 0)],
    "many": [("fb"[i % 2], (i * 131) % 5000) for i in range(300)],
    "large": [("f", 30_000_001), ("b", 50_000_000), ("f", 5)],
}


@pytest.mark.parametrize("spec", list(SPECS))
@pytest.mark.parametrize("max_norm", [0.0, 0.01, 1e9, math.inf])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(spec, max_norm, in_place):
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    say("clip", spec, max_norm, in_place)
    grads = clip_inputs(len(spec), SPECS[spec])
    before = [t.clone() for t in grads]
    out = None if in_place else [torch.empty_like(t) for t in grads]
    r = pc.clip_grad_norm(grads, max_norm, out)
    check_clip(before, grads if in_place else out, r, max_norm)
    if max_norm >= 1e9:  # nothing to clip: not a bit changes
        assert all(torch.equal(b, o) for b, o in zip(before, grads if in_place else out))
    if not in_place:
        assert all(torch.equal(b, g) for b, g in zip(before, grads))
        again = [torch.empty_like(t) for t in grads]
        r2 = pc.clip_grad_norm(grads, max_norm, again)
        assert torch.equal(r["norm"], r2["norm"]) and all(torch.equal(a, o) for a, o in zip(again, out))


def test_clip_flat_buffers_of_any_alignment():
    """Tensors that start at every alignment of their type, into places of other alignments; what
    lies between the places is left alone."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    for dt in (torch.float32, torch.bfloat16):
        src = torch.randn(200_000, device="cuda").to(dt)
        dst = torch.full((200_000,), 5.0, device="cuda").to(dt)
        want = dst.clone()
        grads, out, at = [], [], 0
        for i in range(40):
            n = (i * 977) % 4000 + 1
            a, o = at + i % 5, at + (3 * i) % 7
            grads.append(src[a:a + n])
            out.append(dst[o:o + n])
            at += n + 8
        before = [t.clone() for t in grads]
        r = pc.clip_grad_norm(grads, 1.0, out)
        check_clip(before, out, r, 1.0)
        at = 0
        for i, o in enumerate(out):
            want[at + (3 * i) % 7:][:o.numel()] = o
            at += o.numel() + 8
        assert torch.equal(dst, want)


@pytest.mark.parametrize("value", [1e30, 1e-30, 3e38])
def test_clip_range_of_squares(value):
    """Squares beyond float's range, either way."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    g = [torch.full((1000,), value, device="cuda"), torch.full((10,), value, device="cuda").to(torch.bfloat16)]
    before = [t.clone() for t in g]
    exact = math.sqrt(sum(float(t.double().square().sum()) for t in before))
    r = pc.clip_grad_norm(g, 1.0)
    assert float(r["norm"]) == pytest.approx(exact, rel=1e-6) if exact < 3.4e38 else math.isinf(float(r["norm"]))
    s = min(1.0, 1.0 / (exact + 1e-6))
    assert torch.allclose(g[0].double(), before[0].double() * s, rtol=2.0 ** -22, atol=0)


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_norm_not_finite(bad, in_place):
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    g = clip_inputs(3, [("f", 5000), ("b", 777)])
    g[1][700] = bad
    before = [t.clone() for t in g]
    out = None if in_place else [torch.empty_like(t) for t in g]
    r = pc.clip_grad_norm(g, 0.5, out)
    assert not math.isfinite(float(r["norm"])) and float(r["scale"]) == 1.0
    for b, o in zip(before, g if in_place else out):
        assert torch.equal(torch.nan_to_num(b, 9.0), torch.nan_to_num(o, 9.0))


def test_clip_refusals_and_graph():
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    x = torch.ones(8, 4, device="cuda")
    for grads, out in (([x.t()], None), ([x.half()], None), ([x], []), ([x], [x.bfloat16()]), ([x], [x[:4]]), ([x, x.cpu()], None)):
        with pytest.raises(pc.PrunedCTCError):
            pc.clip_grad_norm(grads, 1.0, out)
    with pytest.raises(pc.PrunedCTCError):
        pc.clip_grad_norm([x], -1.0)
    g = clip_inputs(5, [("f", 70_000), ("b", 3000)])
    pc.clip_grad_norm([t.clone() for t in g], 1.0)
    out = [torch.empty_like(t) for t in g]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = pc.clip_grad_norm(g, 1.0, out)
    for i in range(4):
        for t in g:
            t.mul_(1.5)
        graph.replay()
        torch.cuda.synchronize()
        check_clip(g, out, r, 1.0)
        torch.randn(1000, device="cuda").sum().item()


def test_clip_head_gradients():
    """A training step's use: the fused call's gradients, clipped together."""
    from paper_2609_33645_amd import prunedctc as pc
    from paper_2609_33645_amd import workloads
    from tests.gpu_util import to_dev
    wl = workloads.random_small(5, N=4, T_range=(10, 40), D=64, V=1000, dtype="bf16")
    H, W, y = to_dev(wl)
    out = pc.pruned_ctc_fwd_bwd(H, W, y, wl.input_lengths, wl.target_lengths, wl.blank, want_db=True)
    grads = [out["dW"], out["db"], out["dH"]]
    before = [t.clone() for t in grads]
    r = pc.clip_grad_norm(grads, 1.0)
    check_clip(before, grads, r, 1.0)
    assert float(pc.clip_grad_norm(grads, math.inf)["norm"]) == pytest.approx(1.0, rel=1e-5)


def test_fit_and_decode_example():
    """The example end to end: the loss falls, and every beam's predictor state, reordered through all
    of its frames, is the one its labels define (sums of at most 80 vectors in another order)."""
    from paper_2609_33645_amd import fit_and_decode
    r = fit_and_decode.run(steps=120, beams=4, classes=100, N=6)
    say(r)
    assert r["loss_last"] < 0.1 * r["loss_first"] and 0 < r["norm_last"] < r["norm_max"]
    assert r["errors best of beams"] <= r["errors beam"] < r["labels"]
    assert r["predictor off by"] < 1e-4
