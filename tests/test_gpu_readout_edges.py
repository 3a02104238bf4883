"""Readout with beams and clipping on the GPU, where calls are out of the ordinary (references and
tolerances as in test_gpu_readout)."""
import numpy as np
import pytest

from tests import readout_ref as ref
from tests.gpu_util import say
from tests.test_gpu_readout import check_result, random_frames, run_search

pytestmark = pytest.mark.gpu


# ---- rows with empty places ------------------------------------------------------------------

def with_gaps(seed, ids, lp, share):
    """The rows with places made empty in every way, whole runs at the beginning among them; and the same
    rows with the empty places last."""
    r = np.random.default_rng(seed)
    ids, lp = ids.copy(), lp.copy()
    T, C = ids.shape
    gone = r.random((T, C)) < share
    for t in range(0, T, 3):
        gone[t, :r.integers(0, C)] = True
    gone[T // 2] = False
    kind = r.integers(0, 4, size=(T, C))
    ids[gone & (kind == 0)] = -1
    ids[gone & (kind == 1)] = -7
    lp[gone & (kind == 2)] = -np.inf
    lp[gone & (kind == 3)] = np.nan
    order = np.argsort(gone, 1, kind="stable")
    packed = np.sort(gone, 1)
    return ids, lp, np.where(packed, -1, np.take_along_axis(ids, order, 1)), \
        np.where(packed, -np.inf, np.take_along_axis(lp, order, 1)).astype(np.float32)


@pytest.mark.parametrize("K,C", [(1, 3), (1, 64), (4, 8), (8, 16), (8, 64), (16, 24), (32, 40), (32, 64)])
@pytest.mark.parametrize("share", [0.1, 0.6])
def test_search_empty_places(K, C, share):
    """An empty place is no candidate wherever it stands: rows with them are searched bit for bit as the rows
    without them, and as the definition has it."""
    say("empty places", K, C, share)
    parts, packed, T = [], [], (1, 9, 30)
    for n, t in enumerate(T):
        for k in range(400):
            ids, lp, bl = random_frames(100 * n + 7919 * k + K, t, C, C + 6)
            a, b, c, d = with_gaps(k, ids, lp, share)
            s = ref.Search(K).run(a, b, bl)
            if s.gap > 2e-5:
                break
        parts.append((a, b, bl, s))
        packed.append((c, d, bl))
    got, same = run_search([q[:3] for q in parts], K), run_search(packed, K)
    assert all(np.array_equal(got[k], same[k]) for k in got)
    for n, q in enumerate(parts):
        assert q[3].gap > 2e-5
        check_result(got, n, q[3].result(), T[n])


def test_search_empty_places_first():
    """Candidates behind more empty places than there are beams."""
    def one(K, ids, lp, bl):
        ids, lp, bl = np.array([ids], np.int32), np.array([lp], np.float32), np.array([bl], np.float32)
        check_result(run_search([(ids, lp, bl)], K), 0, ref.Search(K).run(ids, lp, bl).result(), 1)
    one(1, [-1, -1, 9], [-.01, -.02, -.05], -4.0)
    one(4, [-1] * 6 + [7, 8], [-.1 * k for k in range(1, 9)], -3.0)
    one(2, [5, 6, 4, 7], [-np.inf, np.nan, -0.5, -1.0], -3.0)


@pytest.mark.parametrize("K", [1, 3, 8, 32])
def test_search_empty_places_of_offered_classes(K):
    """An empty place may hold a class that the row offers in another place."""
    parts = []
    for seed in range(6):
        for k in range(400):
            ids, lp, bl = random_frames(1000 * seed + k, 20, 8, 9)
            r = np.random.default_rng(k)
            for t in range(20):  # 4 of 8 places empty, with the classes of the others, scores gone
                gone = np.sort(r.choice(8, 4, replace=False))
                ids[t, gone] = ids[t, np.setdiff1d(np.arange(8), gone)]
                lp[t, gone] = r.choice([-np.inf, np.nan], 4)
            s = ref.Search(K)
            for t in range(20):
                keep = lp[t] > -np.inf
                s.step(ids[t][keep], lp[t][keep], bl[t])
            if s.gap > 2e-5:
                break
        parts.append((ids, lp, bl, s))
    got = run_search([q[:3] for q in parts], K)
    for n, q in enumerate(parts):
        assert q[3].gap > 2e-5
        check_result(got, n, q[3].result(), 20)


# ---- equal totals ------------------------------------------------------------------------------

@pytest.mark.parametrize("K", [1, 2, 4, 7, 8, 16, 31, 32])
@pytest.mark.parametrize("C", [1, 6, 64])
@pytest.mark.parametrize("bonus", [0.0, -0.5, 0.25])
def test_search_ties(K, C, bonus):
    """Equal totals go by their order: beams that stay, then grown ones by beam and class.  Every frame has
    classes of its own and scores of a few halves, so that all sums are exact."""
    say("ties", K, C, bonus)
    parts = []
    for seed, T in ((1, 1), (2, 3), (3, 12), (4, 12)):
        r = np.random.default_rng(seed + K)
        ids = 1 + np.arange(T * C, dtype=np.int32).reshape(T, C)
        lp = -np.sort(r.integers(1, 4, size=(T, C)) / 2.0, 1).astype(np.float32)
        parts.append((ids, lp, -(r.integers(1, 4, size=T) / 2.0).astype(np.float32)))
    got = run_search(parts, K, bonus)
    for n, q in enumerate(parts):
        check_result(got, n, ref.Search(K, bonus).run(*q).result(), len(q[2]), tol=0.0)


# ---- scores near float's lowest value ------------------------------------------------------------

def test_search_scores_near_the_lowest_value():
    """Masks of large finite scores: a total far below any other is still above -inf, and its prefix stays, also
    where masses are added (a beam's last label is offered).  Every sum has one term above the others' last bits."""
    f = np.float32
    low = float(np.finfo(f).min)

    def one(K, rows):
        ids, lp, bl = (np.array([r[i] for r in rows], d) for i, d in ((0, np.int32), (1, f), (2, f)))
        want = ref.Search(K).run(ids, lp.astype(np.float64), bl.astype(np.float64)).result()
        got = run_search([(ids, lp, bl)], K)
        check_result(got, 0, want, len(rows), tol=1e-6 * max(1.0, *(abs(s) for _, s in want)))
    one(1, [([5], [-0.5], -50.0), ([5], [-2e38], -3e38)])             # its label, then blank far below
    one(1, [([5], [-0.5], -50.0), ([5], [-3e38], -2e38)])             # the other way
    one(1, [([5], [-0.5], -50.0), ([5], [low], low), ([5], [-1.0], -9.0)])
    one(2, [([5, 6], [-1.0, -1e31], -1e33), ([5, 6], [-1e32, -2e35], -3e34)])
    one(4, [([5, 6], [-1.0, -1e33], -1e31), ([5, 6], [-0.5, -1e36], -1e34)])


# ---- replays -------------------------------------------------------------------------------------

@pytest.mark.parametrize("K", [2, 4])
def test_result_after_replays_at_another_position(K):
    """One captured advance replayed frame after frame writes over its own nodes: the labels are unspecified, but
    the lengths stay in bounds, nothing outside the state is read, and a reset makes the search right again."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    say("replays", K)
    N, C, T = 3, 6, 50
    parts = [random_frames(70 + n, T, C, 9) for n in range(N)]
    frames = [torch.from_numpy(np.stack([q[i] for q in parts], 1)).cuda() for i in range(3)]
    now = [f[0].clone() for f in frames]
    b = pc.BeamSearch(N, K, T)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.advance(*now, [1] * N)
    for t in range(T):
        for x, f in zip(now, frames):
            x.copy_(f[t])
        graph.replay()
        torch.cuda.synchronize()
    r = b.result(T)
    lengths = r["token_lengths"].cpu().numpy()
    assert lengths.min() >= -1 and lengths.max() <= T
    past = np.arange(T)[None, None, :] >= lengths[:, :, None]
    assert (r["tokens"].cpu().numpy()[past] == -1).all()
    b.reset()
    b.advance(*(torch.cat([f[:, n] for n in range(N)]) for f in frames), [T] * N)
    got = {k: v.cpu().numpy() for k, v in b.result(T).items()}
    want = run_search(parts, K)
    assert all(np.array_equal(got[k], want[k]) for k in want)
    # more replays than the state has room for frames
    small = pc.BeamSearch(N, K, 5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        small.advance(*now, [1] * N)
    for t in range(T):
        for x, f in zip(now, frames):
            x.copy_(f[t])
        graph.replay()
        torch.cuda.synchronize()
    assert int(small.result(5)["token_lengths"].max()) <= 5


def test_long_prefix_cut_at_segments():
    """The labels hang together in segments of 16: cuts on both sides of a segment's edge, and of 63 segments'."""
    T = 1100
    path = np.random.default_rng(1).integers(1, 500, size=T) * 2
    path[1:] += (path[1:] == path[:-1])
    ids = np.stack([path, path + 2000], 1).astype(np.int32)
    lp = np.tile(np.array([[-0.01, -9.0]], np.float32), (T, 1))
    bl = np.full(T, -12.0, np.float32)
    for n in (15, 16, 17, 1007, 1008, 1009, 1100):
        for cut in sorted({min(n, c) for c in (15, 16, 17, 1008, n)}):
            got = run_search([(ids[:n], lp[:n], bl[:n])], 1, max_frames=T, max_tokens=cut)
            assert got["tokens"][0, 0].tolist() == path[:cut].tolist() and got["token_lengths"][0, 0] == n


# ---- other streams -------------------------------------------------------------------------------

def test_other_stream_keeps_a_search_and_iterators_tensors():
    """A search let go of right after its calls on a busy stream, and gradients that came as an iterator: their
    memory, asked for again on the current stream, is not handed out before the work is done."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    parts = [random_frames(n, 40, 6, 9) for n in range(4)]
    want = run_search(parts, 8, max_frames=40, max_tokens=40)
    cat = [torch.from_numpy(np.concatenate([q[i] for q in parts])).cuda() for i in range(3)]
    grads = [torch.randn(300_000, device="cuda") for _ in range(3)]
    norm = pc.clip_grad_norm(grads, 1.0, out=[torch.empty_like(g) for g in grads])["norm"].clone()
    a = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    for _ in range(3):
        b, gs = pc.BeamSearch(4, 8, 40), [g.clone() for g in grads]
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(4):
                torch.mm(a, a)
        b.advance(*cat, [40] * 4, stream=side)
        got = b.result(40, stream=side)
        clipped = pc.clip_grad_norm((g for g in gs), 1.0, out=(torch.empty_like(g) for g in grads), stream=side)
        nbytes = b._state.untyped_storage().nbytes()
        del b, gs
        junk = [torch.full((nbytes,), 7, dtype=torch.uint8, device="cuda"),
                *(torch.full((300_000,), 7.0, device="cuda") for _ in range(3))]
        torch.cuda.synchronize()
        assert all(np.array_equal(want[k], got[k].cpu().numpy()) for k in want)
        assert torch.equal(clipped["norm"], norm)
        del junk


# ---- numbers of frames ---------------------------------------------------------------------------

def test_numbers_of_frames_that_no_call_takes():
    """Numbers that are not whole, or that int32 does not hold, are refused where they would have been cut off to
    numbers that fit the candidates."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    ids, lp, bl = (torch.from_numpy(x).cuda() for x in random_frames(1, 3, 4, 6))
    b = pc.BeamSearch(2, 4, 10)
    for frames, code in (([1.7, 2.0], -1), ([2 ** 32 + 1, 2], -3), (np.array([2 ** 32 + 1, 2]), -3),
                         (torch.tensor([1.0, 2.0]), -1), ([1, 2, 0], -1), ([-1, 4], -3), (np.array([1.0, 2.0]), -1)):
        with pytest.raises(pc.PrunedCTCError) as e:
            b.advance(ids, lp, bl, frames)
        assert e.value.code == code, frames
    assert b.frames_done.tolist() == [0, 0]
    first = b.advance(ids, lp, bl, [1, 2])
    for frames in ((1, 2), np.array([1, 2]), torch.tensor([1, 2], device="cuda"), np.array([1, 2], np.int32)):
        b.reset()
        assert torch.equal(b.advance(ids, lp, bl, frames), first) and b.frames_done.tolist() == [1, 2]
    H, W = torch.randn(3, 64, device="cuda"), torch.randn(9, 64, device="cuda")
    for lengths, code in (([1.5, 2.9], -1), (np.array([2 ** 32 + 1, 2]), -3), ([0, 3], -3), ([3, 1], -1)):
        with pytest.raises(pc.PrunedCTCError) as e:
            pc.beam_decode(H, W, lengths)
        assert e.value.code == code, lengths
    for lengths in ([1, 2], torch.tensor([1, 2])):
        assert pc.beam_decode(H, W, lengths)["token_lengths"].shape == (2, 8)


# ---- lists whose tensors overlap -----------------------------------------------------------------

def test_clip_overlapping_tensors():
    """What the order of the work would decide is refused; what it would not is done."""
    import math

    import torch

    from paper_2609_33645_amd import prunedctc as pc
    flat = torch.randn(1000, device="cuda")
    a, b, mid = flat[:400], flat[400:], flat[100:600]
    spare = torch.empty(2000, device="cuda")
    before = flat.clone()
    for grads, out in (([a, b, a], None), ([a, mid], None), ([a, b], [spare[:400], spare[399:999]]),
                       ([a, b], [flat[:400], flat[399:999]]), ([a, b], [b[:400], spare[:600]]), ([a], [flat[1:401]])):
        with pytest.raises(pc.PrunedCTCError) as e:
            pc.clip_grad_norm(grads, 1.0, out)
        assert e.value.code == -1
    assert torch.equal(flat, before)
    # read twice: counted twice, written apart
    r = pc.clip_grad_norm([a, mid, a], 1.0, [spare[:400], spare[400:900], spare[900:1300]])
    exact = math.sqrt(sum(float(t.double().square().sum()) for t in (a, mid, a)))
    assert float(r["norm"]) == pytest.approx(exact, rel=2.0 ** -23)
    s = 1.0 / (exact + 1e-6)
    assert torch.allclose(spare[:1300].double(), torch.cat([a, mid, a]).double() * s, rtol=2.0 ** -22, atol=0)
    assert float(pc.clip_grad_norm([a, a], math.inf)["norm"]) == pytest.approx(
        math.sqrt(2 * float(a.double().square().sum())), rel=2.0 ** -23) and torch.equal(flat, before)
    # out that are the gradients themselves, some of them
    pc.clip_grad_norm([a, b], 1.0, [a, spare[:600]])
    s = 1.0 / (float(before.double().norm()) + 1e-6)
    assert torch.allclose(torch.cat([a, spare[:600]]).double(), before.double() * s, rtol=2.0 ** -22, atol=0)
    assert torch.equal(b, before[400:])


def test_reorder_overlapping_tensors():
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    N, K = 2, 4
    flat = torch.arange(3 * N * K * 5, device="cuda").float()
    parents = torch.tensor([[1, 0, 3, 3], [2, 2, 2, 0]], dtype=torch.int32, device="cuda")
    at = lambda i, x=flat: x[i:i + N * K * 5].view(N, K, 5)  # noqa: E731
    a, b, c, mid = at(0), at(40), at(80), at(20)
    spare = torch.zeros_like(flat)
    before = flat.clone()
    for states, out in (([a, a], None), ([a, b, mid], None), ([a, b], [c, c]), ([a, b], [c, at(79)]), ([a, b], [b, a]),
                        ([a], [at(1)]), ([a, b, c], [a, b, mid])):
        with pytest.raises(pc.PrunedCTCError) as e:
            pc.beam_reorder(states, parents, out)
        assert e.value.code == -1
    assert torch.equal(flat, before)
    want = [torch.stack([x[n][parents[n].long()] for n in range(N)]) for x in (a, mid)]
    got = pc.beam_reorder([a, mid, a], parents, [at(0, spare), at(40, spare), at(80, spare)])
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[0])
    got = pc.beam_reorder([a, b], parents, [a, at(0, spare)])  # in place and not
    assert got[0] is a and torch.equal(a, want[0])
    assert torch.equal(got[1], torch.stack([b[n][parents[n].long()] for n in range(N)]))


def test_reorder_beside_its_parents():
    """States that touch the parents' memory without meeting it are reordered; one that meets it is refused."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    flat = torch.zeros(24, dtype=torch.int32, device="cuda")
    before, parents, after = (flat[i:i + 8].view(2, 4) for i in (0, 8, 16))
    parents.copy_(torch.tensor([[3, 2, 1, 0], [1, 1, 0, 0]]))
    for t in (before, after):
        t.copy_(torch.arange(8, device="cuda").view(2, 4))
    pc.beam_reorder([before, after], parents)
    want = torch.tensor([[3, 2, 1, 0], [5, 5, 4, 4]], dtype=torch.int32, device="cuda")
    assert torch.equal(before, want) and torch.equal(after, want)
    for states, out in (([parents], None), ([flat[4:12].view(2, 4)], None), ([before], [parents])):
        with pytest.raises(pc.PrunedCTCError):
            pc.beam_reorder(states, parents, out)
    assert pc.beam_reorder([parents], parents, [after])[0] is after  # only read
    assert torch.equal(after, torch.tensor([[0, 1, 2, 3], [1, 1, 1, 1]], dtype=torch.int32, device="cuda"))
