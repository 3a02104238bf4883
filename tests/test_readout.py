"""Readout with beams and gradient clipping, without a GPU: the 64-bit reference search against
enumeration of all alignments, and the library's host-side argument checks and sizes."""
import contextlib
import ctypes
import itertools
import math
import os

import numpy as np
import pytest

from tests import readout_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_33645_amd", "libprunedctc.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")


def collapse(path, blank):
    out, prev = [], None
    for c in path:
        if c != prev and c != blank:
            out.append(c)
        prev = c
    return tuple(out)


@pytest.mark.parametrize("T,V,bonus", [(1, 3, 0.0), (3, 3, 0.0), (5, 3, -0.7), (4, 4, 0.3)])
def test_reference_search_is_the_sum_over_alignments(T, V, bonus):
    """With room for every prefix, a prefix's score is the log mass of all alignments that collapse
    to it (Sec. 3.1), plus the bonus of its labels."""
    rng = np.random.default_rng(T * 10 + V)
    z = rng.normal(size=(T, V)) * 2
    ids, logp, blank = ref.candidates(z, V - 1, 0)
    lp = z - np.log(np.exp(z).sum(1, keepdims=True))
    mass = {}
    for path in itertools.product(range(V), repeat=T):
        y = collapse(path, 0)
        mass[y] = mass.get(y, 0.0) + math.exp(sum(lp[t, c] for t, c in enumerate(path)))
    got = dict(ref.Search(10 ** 6, bonus).run(ids, logp, blank).result())
    assert set(got) == set(mass)
    for y, p in mass.items():
        assert got[y] == pytest.approx(math.log(p) + bonus * len(y), abs=1e-12)


def test_reference_search_by_hand():
    """K = 1 on two frames: the better of blank and label a at each frame, then merged mass."""
    s = ref.Search(1)
    s.step([5], [math.log(0.6)], math.log(0.4))
    assert s.result() == [((5,), pytest.approx(math.log(0.6)))]
    s.step([5], [math.log(0.5)], math.log(0.5))
    assert s.result()[0][1] == pytest.approx(math.log(0.6))  # stays by blank and by its label


def _lib():
    import torch  # noqa: F401
    from paper_2609_33645_amd import prunedctc
    return prunedctc.lib()


OK = 0x7f0000000000  # an aligned stand-in; never dereferenced where a check refuses the call


def i32(*xs):
    return np.array(xs, np.int32)


def p(a):
    return a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))


@built
def test_sizes():
    L = _lib()
    up = lambda x: (x + 255) // 256 * 256  # noqa: E731
    assert L.pctc_beam_state_bytes(0, 8, 100) > 0
    for bad in ((-1, 8, 100), (1, 0, 100), (1, 33, 100), (1, 8, -1), (1, 8, 1 << 28), ((1 << 20) + 1, 1, 1)):
        assert L.pctc_beam_state_bytes(*bad) == 0, bad
    # three masses, two hashes and four indices a beam; an offset an utterance; 12 bytes a frame and beam
    nk = 3 * 8
    assert L.pctc_beam_state_bytes(3, 8, 100) == \
        7 * up(nk * 4) + 2 * up(nk * 8) + up(24) + up(nk * 100 * 8) + up(nk * 100 * 4)
    assert L.pctc_clip_workspace_size(-1) == 0 and L.pctc_clip_workspace_size(0) > 0
    c = L.pctc_frame_candidates_workspace_size
    assert c(1, 0, 512, 180_000, 16) > 0
    for bad in ((2, 4, 512, 1000, 16), (1, -1, 512, 1000, 16), (1, 4, 500, 1000, 16), (1, 4, 512, 1, 16),
                (1, 4, 512, 1000, 0), (1, 4, 512, 1000, 65), (1, 4, 512, 524_289, 16)):
        assert c(*bad) == 0, bad
    # the block maxima are held to 512 MiB: more frames take more passes, not more memory (the
    # normaliser's partial sums and a transposed H grow with the frames of a pass alone)
    for D in (512, 4096):
        for dt in (0, 1):
            assert c(dt, 400_000, D, 180_000, 16) == c(dt, 100_000, D, 180_000, 64) \
                < (512 << 20) + 6_144 * (8 * 1030 + 2 * D)
    d = L.pctc_beam_decode_workspace_size
    T = i32(30, 20)
    assert d(1, p(T), 2, 512, 1000, 8, 16) > c(1, 50, 512, 1000, 16)
    assert d(1, p(i32(0, 20)), 2, 512, 1000, 8, 16) == 0
    for bad in ((1, 2, 512, 1000, 0, 16), (1, 2, 512, 1000, 33, 16), (1, 2, 512, 1000, 8, 65), (1, -1, 512, 1000, 8, 16)):
        assert d(bad[0], p(T), *bad[1:]) == 0, bad
    assert d(1, p(T), 0, 512, 1000, 8, 16) > 0


@built
def test_candidates_refusals():
    L = _lib()
    big = 1 << 40

    def call(dt=1, H=OK, M=4, D=64, W=OK, V=100, blank=0, C=8, ids=OK, logp=OK, bl=OK, ws=OK, n=big):
        return L.pctc_frame_candidates(dt, H, M, D, W, None, V, blank, C, ids, logp, bl, ws, n, None)
    for kw in (dict(dt=2), dict(H=OK + 8), dict(W=OK + 8), dict(W=None), dict(H=None), dict(M=-1), dict(D=60), dict(V=1),
               dict(blank=-1), dict(blank=100), dict(C=0), dict(C=65), dict(ids=None), dict(logp=None), dict(bl=None),
               dict(ws=OK + 16)):
        assert call(**kw) == -1, kw
    assert call(ws=None) == -4 and call(n=16) == -4
    assert call(M=0, H=None, ids=None, logp=None, bl=None, ws=None) == 0


@built
def test_beam_refusals():
    L = _lib()
    big = 1 << 40
    done = i32(0, 95)

    def adv(ids=OK, logp=OK, bl=OK, C=8, frames=i32(3, 4), N=2, K=4, cap=100, bonus=0.0, dn=done, state=OK, n=big):
        at = lambda a: None if a is None else a.ctypes.data  # noqa: E731
        return L.pctc_beam_advance(ids, logp, bl, C, at(frames), N, K, cap, bonus, at(dn), state, n, None, None)
    for kw in (dict(ids=None), dict(logp=None), dict(bl=None), dict(C=0), dict(C=65), dict(N=-1), dict(K=0), dict(K=33),
               dict(cap=-1), dict(bonus=math.nan), dict(bonus=math.inf), dict(frames=None), dict(dn=None),
               dict(state=OK + 16)):
        assert adv(**kw) == -1, kw
    assert adv(state=None) == -4 and adv(n=64) == -4
    for frames in (i32(-1, 2), i32(3, 6), i32(101, 0), i32(0, 2 ** 31 - 1)):
        assert adv(frames=frames) == -3, frames
    assert adv(dn=i32(-1, 0)) == -3
    assert done.tolist() == [0, 95]  # refused calls count no frames
    assert adv(N=0, frames=None, dn=None, state=None) == 0
    assert L.pctc_beam_reset(2, 4, 100, None, big, None) == -4 and L.pctc_beam_reset(2, 40, 100, OK, big, None) == -1
    assert L.pctc_beam_reset(0, 4, 100, None, 0, None) == 0

    def res(N=2, K=4, cap=100, state=OK, n=big, mt=10, tokens=OK, lengths=OK, scores=OK):
        return L.pctc_beam_result(N, K, cap, state, n, mt, tokens, lengths, scores, None)
    for kw in (dict(mt=-1), dict(tokens=None), dict(lengths=None), dict(scores=None), dict(K=0), dict(state=OK + 8)):
        assert res(**kw) == -1, kw
    assert res(state=None) == -4 and res(N=0, state=None) == 0


@built
def test_decode_refusals():
    L = _lib()
    T = i32(30, 20)

    def call(dt=1, H=OK, D=64, W=OK, V=100, T=T, N=2, blank=0, K=4, C=8, bonus=0.0, mt=10, tokens=OK, lengths=OK,
             scores=OK, ws=OK, n=1 << 40):
        return L.pctc_beam_decode(dt, H, D, W, None, V, p(T) if T is not None else None, N, blank, K, C, bonus, mt, tokens,
                                  lengths, scores, None, None, None, ws, n, None)
    for kw in (dict(dt=3), dict(H=None), dict(H=OK + 4), dict(D=0), dict(W=None), dict(V=1), dict(T=None), dict(N=-1),
               dict(blank=100), dict(K=0), dict(K=33), dict(C=0), dict(C=65), dict(bonus=math.nan), dict(mt=-1),
               dict(tokens=None), dict(lengths=None), dict(scores=None), dict(ws=OK + 64)):
        assert call(**kw) == -1, kw
    assert call(T=i32(0, 4)) == -3 and call(ws=None) == -4 and call(n=100) == -4
    assert call(N=0, T=None) == 0


@built
def test_reorder_and_clip_refusals():
    L = _lib()
    vp = lambda *xs: (ctypes.c_void_p * max(len(xs), 1))(*xs)  # noqa: E731
    i64 = lambda *xs: (ctypes.c_int64 * max(len(xs), 1))(*xs)  # noqa: E731
    r = L.pctc_beam_reorder
    assert r(-1, vp(OK), None, i64(4), OK, 2, 4, None) == -1
    assert r(1, None, None, i64(4), OK, 2, 4, None) == -1 and r(1, vp(OK), None, None, OK, 2, 4, None) == -1
    assert r(1, vp(OK), None, i64(-4), OK, 2, 4, None) == -1 and r(1, vp(None), None, i64(4), OK, 2, 4, None) == -1
    assert r(1, vp(OK), vp(None), i64(4), OK, 2, 4, None) == -1 and r(1, vp(OK), None, i64(4), None, 2, 4, None) == -1
    assert r(1, vp(OK), None, i64(4), OK, 2, 0, None) == -1 and r(1, vp(OK), None, i64(4), OK, 2, 33, None) == -1
    assert r(1, vp(OK), None, i64((1 << 36) + 1), OK, 2, 4, None) == -1
    assert r(0, None, None, None, None, 2, 4, None) == 0 and r(1, vp(None), None, i64(0), None, 2, 4, None) == 0
    assert r(1, vp(OK), None, i64(4), None, 0, 4, None) == 0
    c = L.pctc_clip_grad_norm
    f32, bf = (ctypes.c_int32 * 1)(0), (ctypes.c_int32 * 1)(1)
    big = 1 << 30
    assert c(-1, vp(OK), None, i64(4), f32, 1.0, OK, None, OK, big, None) == -1
    for bad in (math.nan, -1.0):
        assert c(1, vp(OK), None, i64(4), f32, bad, OK, None, OK, big, None) == -1
    assert c(1, vp(OK), None, i64(4), f32, 1.0, None, None, OK, big, None) == -1
    assert c(1, None, None, i64(4), f32, 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(OK), None, i64(4), (ctypes.c_int32 * 1)(2), 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(OK), None, i64(-1), f32, 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(OK), None, i64((1 << 34) + 1), f32, 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(None), None, i64(4), f32, 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(OK), vp(None), i64(4), f32, 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(OK + 2), None, i64(4), f32, 1.0, OK, None, OK, big, None) == -1  # off its type's alignment
    assert c(1, vp(OK), vp(OK + 1), i64(4), bf, 1.0, OK, None, OK, big, None) == -1
    assert c(1, vp(OK), None, i64(4), f32, 1.0, OK, None, None, big, None) == -4
    assert c(1, vp(OK), None, i64(4), f32, 1.0, OK, None, OK, 16, None) == -4
    assert c(1, vp(OK), None, i64(4), f32, 1.0, OK, None, OK + 8, big, None) == -1


@built
def test_binding_refusals():
    """The binding refuses what it can see without a device."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    x = torch.zeros(4, 8)
    for call in (lambda: pc.frame_candidates(x, x, 2), lambda: pc.beam_decode(x, x, [4]),
                 lambda: pc.clip_grad_norm([x], 1.0), lambda: pc.clip_grad_norm([], 1.0),
                 lambda: pc.beam_reorder([x], torch.zeros(2, 2, dtype=torch.int32)),
                 lambda: pc.frame_candidates(x.half(), x.half(), 2)):
        with pytest.raises(pc.PrunedCTCError) as e:
            call()
        assert e.value.code == -1


@built
@pytest.mark.parametrize("dtype", [0, 1])
def test_candidates_passes_stay_in_the_workspace(dtype):
    """Every pass of a call uses no more than the workspace asked for: short and long vocabularies, narrow and
    wide heads, and numbers of frames whose last pass is short while a full one is too large to be transposed."""
    L = _lib()
    frames = ctypes.c_int32()

    def check(M, D, V, C):
        size, m0, n = L.pctc_frame_candidates_workspace_size(dtype, M, D, V, C), 0, 0
        assert size > 0
        while m0 < M:
            used = L.pctc_frame_candidates_pass(dtype, M, D, V, C, m0, ctypes.byref(frames))
            assert 0 < used <= size and 0 < frames.value <= M - m0, (M, D, V, C, m0, frames.value, used - size)
            m0, n = m0 + frames.value, n + 1
        return n
    assert check(252_500, 8192, 512, 8) == 2 and check(168_000, 8192, 768, 8) == 2
    assert check(270_000, 5120, 512, 8) == 2
    for D in (8, 128, 512, 640, 4096, 8192, 65_536, 1 << 20):
        for V in (2, 300, 512, 768, 5000, 32_768, 180_000, 524_288):
            for C in (1, 16, 64):
                full = ctypes.c_int32()
                assert L.pctc_frame_candidates_pass(dtype, 1 << 30, D, V, C, 0, ctypes.byref(full)) > 0
                F = full.value
                for M in (1, 63, F - 1, F, F + 1, F + 100, F + F // 16, F + F // 2, 2 * F, 2 * F + 3000, 5 * F + 7):
                    check(M, D, V, C)
    for bad in ((1, 512, 1000, 16, 1), (1, 512, 1000, 16, -1), (0, 512, 1000, 16, 0), (4, 500, 1000, 16, 0)):
        assert L.pctc_frame_candidates_pass(dtype, *bad, ctypes.byref(frames)) == 0
    assert L.pctc_frame_candidates_pass(dtype, 4, 512, 1000, 16, 0, None) == 0


def test_kernels_go_to_the_tensors_device(monkeypatch):
    """Calls without a device: a call whose tensors are on another device than the current one launches with
    theirs current, on its current stream, and leaves the device as it was, also where it fails; a stream of
    another device is refused."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    now, log = [0], []
    monkeypatch.setattr(pc, "_current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "set_device", lambda d: now.__setitem__(0, d))
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 100 + d)

    class Context:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            self.was, now[0] = now[0], self.stream.device.index

        def __exit__(self, *error):
            now[0] = self.was
    monkeypatch.setattr(torch.cuda, "stream", Context)

    @pc._asynchronous
    def launch(index, fail=False):
        handle = pc._raw_stream(torch.device("cuda", index))
        log.append((now[0], handle))
        if fail:
            raise ValueError
        return handle

    @pc._asynchronous
    def outer(index):
        return launch(index) + launch(index)
    for index in (0, 1, 3):
        assert launch(index) == 100 + index and now == [0]
        assert outer(index) == 200 + 2 * index and now == [0]
        with pytest.raises(ValueError):
            launch(index, fail=True)
        assert now == [0]
    assert all(handle == 100 + device for device, handle in log) and {device for device, _ in log} == {0, 1, 3}

    class Stream:
        device = torch.device("cuda", 1)
    assert launch(1, stream=Stream()) == 101 and now == [0]
    with pytest.raises(pc.PrunedCTCError) as e:
        launch(0, stream=Stream())
    assert e.value.code == -1 and now == [0] and launch(2) == 102 and now == [0]


@built
def test_search_on_no_gpu_is_refused():
    from paper_2609_33645_amd import prunedctc as pc
    with pytest.raises(pc.PrunedCTCError) as e:
        pc.BeamSearch(1, 4, 10, device="cpu")
    assert e.value.code == -1


def test_tensors_of_a_call_on_a_stream_are_kept(monkeypatch):
    """Every device tensor that a call on a given stream works on is told to the allocator: single ones, those
    of lists, of iterables of any kind (which the call still gets whole), and a search's own state."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc

    class Device(torch.Tensor):
        is_cuda = True

        def record_stream(self, stream):
            kept.append((self.mark, stream))

    class Holder:
        pass

    def tensor(mark):
        t = torch.zeros(1).as_subclass(Device)
        t.mark = mark
        return t
    kept, seen = [], []
    monkeypatch.setattr(torch.cuda, "stream", contextlib.nullcontext)

    @pc._asynchronous
    def call(*args, **kw):
        seen.extend(len(list(a)) for a in args if not isinstance(a, Holder))
    one, search = tensor(0), Holder()
    search._state = tensor(1)
    listed = {2: tensor(2), 3: tensor(3)}
    call(search, one, [tensor(4)], (tensor(5),), listed.values(), (tensor(k) for k in (6, 7)), iter([tensor(8)]),
         out=iter([tensor(9)]), stream="side")
    assert sorted(k for k, _ in kept) == list(range(10)) and {s for _, s in kept} == {"side"}
    assert seen == [1, 1, 1, 2, 2, 1]


def test_numbers_of_frames_are_taken_as_they_are():
    """Whole numbers of any integer type and container; a number that int32 does not hold, or that is no whole
    one, is refused and not cut off."""
    import torch

    from paper_2609_33645_amd import prunedctc as pc
    for x in ([3, 0, 7], (3, 0, 7), np.array([3, 0, 7]), np.array([3, 0, 7], np.int32), np.array([3, 0, 7], np.uint8),
              torch.tensor([3, 0, 7]), [np.int64(3), np.int32(0), 7], np.array([[3, 0, 7]] * 2, np.int32).T[:, 0],
              np.array([3, 9, 0, 9, 7], np.int32)[::2]):
        assert list(pc._counts(x)) == [3, 0, 7]
    assert len(pc._counts([])) == 0 and len(pc._counts(np.zeros(0))) == 0
    assert list(pc._counts([-1])) == [-1]  # (refused where lengths are)
    for x, code in (([1.7], -1), (np.array([2.0]), -1), (torch.tensor([1.0]), -1), ([2 ** 32], -3), ([2 ** 31], -3),
                    (np.array([2 ** 32 + 1]), -3), (torch.tensor([2 ** 40]), -3), (5, -1), (None, -1), ([None], -1),
                    (np.array([[1], [2]], np.int32), -1), (np.int32(4), -1)):
        with pytest.raises(pc.PrunedCTCError) as e:
            pc._counts(x)
        assert e.value.code == code, x


@built
def test_clip_refuses_overlaps():
    """Memory that would be written beside another reader or writer of the list is refused before any work;
    the calls that are in order get as far as their missing workspace."""
    L = _lib()

    def call(grads, n, out=None, dtypes=None, max_norm=1.0):
        vp = lambda xs: (ctypes.c_void_p * len(xs))(*xs)  # noqa: E731
        k = len(grads)
        return L.pctc_clip_grad_norm(k, vp(grads), None if out is None else vp(out), (ctypes.c_int64 * k)(*n),
                                     (ctypes.c_int32 * k)(*(dtypes or [0] * k)), max_norm, OK, None, None, 0, None)
    A, B, C = OK, OK + 400, OK + 800  # 100 float32 values apart
    fine, refused = -4, -1
    assert call([A, B, C], [100, 100, 100]) == fine and call([C, A, B], [100, 100, 100]) == fine
    assert call([A], [100]) == fine and call([A, A], [100, 0]) == fine and call([A, None], [100, 0]) == fine
    assert call([A, B, A], [100, 100, 100]) == refused  # the same gradient twice
    assert call([C, A, B], [100, 101, 100]) == refused and call([B, A], [50, 100 + 1]) == refused
    assert call([A, A + 200], [100, 100], dtypes=[1, 1]) == fine and call([A, A + 200], [101, 100], dtypes=[1, 1]) == refused
    assert call([A, A], [100, 100], max_norm=math.inf) == fine  # nothing is written
    # other tensors to write to
    D, E, F = OK + 4000, OK + 4400, OK + 4800
    assert call([A, A, B], [100, 100, 100], out=[D, E, F]) == fine  # read twice, written apart
    assert call([A, B, C], [100] * 3, out=[A, B, C]) == fine and call([C, A, B], [100] * 3, out=[C, A, B]) == fine
    assert call([A, B, C], [100] * 3, out=[F, B, D]) == fine
    for out in ([D, D, F], [D, D + 4, F], [B, A, C], [A + 4, D, E], [D, E, A], [D, E, C + 396], [D, E, A + 796]):
        assert call([A, B, C], [100] * 3, out=out) == refused, out
    assert call([A], [100], out=[A + 4]) == refused and call([A], [100], out=[A]) == fine
    assert call([A, B], [100, 100], out=[D, D], max_norm=math.inf) == refused  # copies are written
    # against a plain search of all pairs
    rng = np.random.default_rng(0)
    seen = set()
    for _ in range(4000):
        k = int(rng.integers(1, 5))
        n = rng.integers(0, 4, size=k)
        g = rng.integers(0, 24, size=k)
        o = None if rng.random() < 0.4 else np.where(rng.random(k) < 0.3, g, rng.integers(0, 24, size=k))
        w = g if o is None else o
        meet = lambda a, b, i, j: a < b + n[j] and b < a + n[i] and n[i] > 0 and n[j] > 0  # noqa: E731
        bad = any(meet(w[i], w[j], i, j) for i in range(k) for j in range(i)) or (
            o is not None and any(meet(o[i], g[j], i, j) and (i != j or o[i] != g[j]) for i in range(k) for j in range(k)))
        seen.add(bad)
        got = call([OK + 4 * int(x) for x in g], n.tolist(), None if o is None else [OK + 4 * int(x) for x in o])
        assert got == (refused if bad else fine), (n, g, o)
    assert seen == {False, True}


@built
def test_reorder_refuses_overlaps():
    """A state twice in a list that is reordered in place, or an out that overlaps another tensor."""
    L = _lib()

    def refused(states, sizes, out=None):
        vp = lambda xs: (ctypes.c_void_p * len(xs))(*xs)  # noqa: E731
        k = len(states)
        return L.pctc_beam_reorder(k, vp(states), None if out is None else vp(out), (ctypes.c_int64 * k)(*sizes), OK, 2, 4,
                                   None) == -1
    A, B, D = OK + 1024, OK + 1024 + 8 * 16, OK + 4096  # two states of 2 x 4 beams of 16 bytes, side by side
    assert refused([A, A], [16, 16]) and refused([A, B], [17, 16]) and refused([B, A, B], [16, 16, 16])
    assert refused([A, B], [16, 16], out=[D, D]) and refused([A, B], [16, 16], out=[D, D + 127])
    assert refused([A, B], [16, 16], out=[B, A]) and refused([A], [16], out=[A + 1])


@built
def test_reorder_refuses_to_write_its_parents():
    L = _lib()
    vp = lambda x: (ctypes.c_void_p * 1)(x)  # noqa: E731

    def refused(state, nbytes, parents, out=None):
        return L.pctc_beam_reorder(1, vp(state), None if out is None else vp(out), (ctypes.c_int64 * 1)(nbytes), parents, 2, 4,
                                   None) == -1
    for at in (0, 4, 124, -28):  # parents of 32 bytes, states of 2 x 4 beams of 16
        assert refused(OK, 16, OK + at)
        assert refused(OK + 4096, 16, OK + at, out=OK)
