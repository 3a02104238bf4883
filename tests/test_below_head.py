"""The operators below the vocabulary head, without a GPU: their references against other definitions, and
the library's host-side argument checks and sizes."""
import os

import numpy as np
import pytest

from tests import below_head_ref as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2609_33645_amd", "libprunedctc.so")
built = pytest.mark.skipif(not os.path.exists(LIB), reason="library not built")
OK = 0x7f0000000000  # a device pointer's stand-in: the calls below end before any device work
BIG = 1 << 40


def _lib():
    import torch  # noqa: F401
    from paper_2609_33645_amd import prunedctc
    return prunedctc.lib()


def test_generator_against_published_words():
    """Philox4x32-10 of counter and key zero, and of all bits set (the authors' known answers)."""
    assert ref.philox([0], 0).tolist() == [[0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]]
    ones = [np.full(1, 0xFFFFFFFF, np.uint64)] * 4
    assert ref._rounds(ones, 0xFFFFFFFF, 0xFFFFFFFF).tolist() == [[0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]]


def test_mask_keeps_its_share():
    for p in (0.1, 0.5):
        n = 1 << 20
        share = ref.kept(n, p, 123, 0).mean()
        assert abs(share - (1 - p)) < 5 * np.sqrt(p * (1 - p) / n) + 2.0 ** -17


@built
def test_dropout_refusals():
    f = _lib().pctc_dropout
    good = dict(dtype=1, x=OK, residual=None, y=OK + BIG, n=100, p=0.1, seed=1, offset=0, dev=None)

    def call(**kw):
        a = dict(good, **kw)
        return f(a["dtype"], a["x"], a["residual"], a["y"], a["n"], a["p"], a["seed"], a["offset"], a["dev"], None)

    assert call(n=0) == 0
    for bad in (dict(dtype=2), dict(n=-1), dict(n=(1 << 34) + 1), dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(x=None),
                dict(y=None), dict(x=OK + 1), dict(y=OK + BIG + 1), dict(residual=OK + 1), dict(y=OK + 2), dict(y=OK + 198),
                dict(residual=OK + BIG + 2), dict(dev=OK + 4), dict(dev=OK + BIG + 8), dict(dtype=0, x=OK + 2)):
        assert call(**bad) == -1, bad


@built
def test_embedding_refusals():
    f = _lib().pctc_embedding
    good = dict(dtype=1, table=OK, V=10, D=8, tokens=OK + BIG, size=4, N=5, scale=1.0, y=OK + 2 * BIG)

    def call(**kw):
        a = dict(good, **kw)
        return f(a["dtype"], a["table"], a["V"], a["D"], a["tokens"], a["size"], a["N"], a["scale"], a["y"], None)

    assert call(N=0) == 0
    for bad in (dict(dtype=3), dict(V=0), dict(V=524_289), dict(D=0), dict(D=(1 << 20) + 1), dict(size=2), dict(N=-1),
                dict(N=(1 << 30) + 1), dict(scale=float("inf")), dict(scale=float("nan")), dict(table=None), dict(tokens=None),
                dict(y=None), dict(table=OK + 1), dict(tokens=OK + BIG + 2), dict(size=8, tokens=OK + BIG + 4), dict(y=OK + 158),
                dict(y=OK + BIG - 78)):
        assert call(**bad) == -1, bad


@built
def test_embedding_backward_refusals_and_sizes():
    lib = _lib()
    f, size = lib.pctc_embedding_backward, lib.pctc_embedding_backward_workspace_size
    assert size(0, 8) >= 0 and size(-1, 8) == size(5, 0) == size((1 << 30) + 1, 8) == 0
    assert size(100, 64) > 0 and size(40_000, 64) > size(20_000, 64) > size(10_000, 64)
    good = dict(dtype=1, dy=OK, tokens=OK + BIG, size=4, N=5, V=10, D=8, scale=1.0, out=0, dW=OK + 2 * BIG, acc=0, ws=OK + 3 * BIG,
                bytes=1 << 30)

    def call(**kw):
        a = dict(good, **kw)
        return f(a["dtype"], a["dy"], a["tokens"], a["size"], a["N"], a["V"], a["D"], a["scale"], a["out"], a["dW"], a["acc"],
                 a["ws"], a["bytes"], None)

    for bad in (dict(dtype=2), dict(out=2), dict(V=0), dict(V=524_289), dict(D=0), dict(size=1), dict(N=-1), dict(scale=float("nan")),
                dict(dy=None), dict(tokens=None), dict(dW=None), dict(dy=OK + 1), dict(dW=OK + 2 * BIG + 2), dict(dW=OK + 76),
                dict(dW=OK + BIG), dict(ws=OK + 3 * BIG + 8), dict(ws=OK + 2 * BIG)):
        assert call(**bad) == -1, bad
    assert call(ws=None) == call(bytes=100) == -4


def test_policy_reference_against_differences():
    rng = np.random.default_rng(3)
    M, D, V = 6, 5, 7
    H, W, b = rng.normal(size=(M, D)), rng.normal(size=(V, D)), rng.normal(size=V)
    t = np.array([0, 3, 6, -1, 2, 2])
    adv, old = rng.normal(size=M), np.full(M, -2.0)
    ref_lp, w = rng.normal(size=M) - 2, rng.random(M)
    f = lambda H, W, b: ref.policy(H, W, b, t, adv, old, ref_lp, w, 0.2, 0.3, 0.1)  # noqa: E731
    r = f(H, W, b)
    assert r["losses"][3] == 0 and not r["dH"][3].any()
    h = 1e-6
    for x, key in ((H, "dH"), (W, "dW"), (b, "db")):
        for i in np.ndindex(x.shape):
            keep = x[i]
            x[i] = keep + h
            up = f(H, W, b)["loss"]
            x[i] = keep - h
            down = f(H, W, b)["loss"]
            x[i] = keep
            # a loss of |L| = 2276 makes about 16 roundings of 2^-53 |L| on each side: 8e-6 over 2 h
            assert abs((up - down) / (2 * h) - r[key][i]) < 1e-7 + 32 * 2.0 ** -53 * abs(r["loss"]) / h, (key, i)


@built
def test_policy_refusals_and_sizes():
    lib = _lib()
    size, f = lib.pctc_policy_workspace_size, lib.pctc_policy_loss
    assert size(1, 100, 64, 300, 0, 1, 0) > size(1, 100, 64, 300, 0, 0, 0) > 0 and size(1, 0, 64, 300, 0, 1, 0) > 0
    for bad in ((2, 1, 64, 300, 0, 1, 0), (1, -1, 64, 300, 0, 1, 0), (1, 1, 60, 300, 0, 1, 0), (1, 1, 0, 300, 0, 1, 0),
                (1, 1, 64, 1, 0, 1, 0), (1, 1, 64, 524_289, 0, 1, 0), (1, 1, 64, 300, 0, 1, 100), (1, 1, 64, 300, 0, 1, -256),
                (1, (1 << 30) + 1, 64, 300, 0, 1, 0)):
        assert size(*bad) == 0, bad
    # the gradients' room does not grow with the vocabulary (chunks differ by up to 10,240 columns of 136 bytes)
    big = [size(1, 4000, 512, V, 0, 1, 0) for V in (150_000, 180_000, 400_000)]
    assert max(big) - min(big) < 2 << 20
    p = [OK + i * BIG for i in range(16)]
    good = dict(dtype=1, H=p[0], M=10, D=64, W=p[1], bias=None, V=300, tokens=p[2], adv=p[3], old=None, ref=None, w=None, lo=0.2,
                hi=0.2, kl=0.0, chunk=0, loss=p[4], losses=p[5], logp=p[6], status=p[7], dH=p[8], dW=p[9], db=None, ws=p[10],
                bytes=1 << 34)

    def call(**kw):
        return f(*dict(good, **kw).values(), None)

    nan, inf = float("nan"), float("inf")
    for bad in (dict(dtype=2), dict(M=-1), dict(D=60), dict(V=1), dict(chunk=100), dict(lo=-0.1), dict(lo=nan), dict(hi=nan),
                dict(hi=-1.0), dict(kl=-0.1), dict(kl=inf), dict(kl=nan), dict(loss=None), dict(W=None), dict(H=None),
                dict(tokens=None), dict(adv=None), dict(losses=None), dict(logp=None), dict(status=None), dict(H=p[0] + 8),
                dict(W=p[1] + 8), dict(dH=p[8] + 8), dict(dW=p[9] + 8), dict(dH=p[0]), dict(dH=p[1] + 16), dict(dW=p[1]),
                dict(dW=p[8] + 1024), dict(ws=p[10] + 16)):
        assert call(**bad) == -1, bad
    # what is written may meet nothing else of the call; floats lie on their size
    full = dict(bias=p[11], old=p[12], ref=p[13], w=p[14], db=p[15])
    for bad in (dict(logp=p[12]), dict(losses=p[3]), dict(losses=p[6] + 36), dict(status=p[2]), dict(loss=p[5] + 32),
                dict(db=p[11]), dict(db=p[9] + 64), dict(losses=p[14]), dict(logp=p[13] + 4), dict(status=p[8] + 4),
                dict(loss=p[4] + 4), dict(logp=p[6] + 2), dict(bias=p[11] + 2), dict(old=p[12] + 1), dict(db=p[15] + 1)):
        assert call(**{**full, **bad}) == -1, bad
    assert call(**full, bytes=1000) == -4  # (nothing else is wrong with it)
    # rows and values whose threads 32 bits would not count
    assert size(1, 1 << 25, 64, 300, 0, 1, 0) > 0 and size(1, (1 << 25) + 1, 64, 300, 0, 1, 0) == 0
    assert size(1, 1 << 23, 1024, 300, 0, 1, 0) > 0 and size(1, (1 << 23) + 1, 1024, 300, 0, 1, 0) == 0


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_ffn_reference_against_differences(act):
    rng = np.random.default_rng(4)
    M, D, F, O = 3, 4, 5, 2
    c = {"x": rng.normal(size=(M, D)), "wg": rng.normal(size=(F, D)), "wu": rng.normal(size=(F, D)), "wd": rng.normal(size=(O, F))}
    dy = rng.normal(size=(M, O))
    r = ref.gated_ffn(*c.values(), act, dy)
    h = 1e-6
    for key, grad in (("x", "dx"), ("wg", "dw_gate"), ("wu", "dw_up"), ("wd", "dw_down")):
        for i in np.ndindex(c[key].shape):
            keep = c[key][i]
            c[key][i] = keep + h
            up = (ref.gated_ffn(*c.values(), act)["y"] * dy).sum()
            c[key][i] = keep - h
            down = (ref.gated_ffn(*c.values(), act)["y"] * dy).sum()
            c[key][i] = keep
            # a sum of magnitude below 100, some 100 roundings of 2^-53 each, over 2 h; truncation below 1e-9
            assert abs((up - down) / (2 * h) - r[grad][i]) < 6e-7, (key, i)


@built
def test_gated_ffn_refusals_and_sizes():
    lib = _lib()
    size = lib.pctc_gated_ffn_workspace_size
    assert size(1, 100, 64, 128, 64, 1) > size(1, 100, 64, 128, 64, 0) > 0 and size(0, 0, 8, 8, 8, 1) > 0
    for bad in ((2, 1, 64, 64, 64, 0), (1, -1, 64, 64, 64, 0), (1, 1, 60, 64, 64, 0), (1, 1, 64, 0, 64, 0), (1, 1, 64, 64, 4, 0),
                (1, (1 << 30) + 1, 64, 64, 64, 0), (1, 1, (1 << 20) + 8, 64, 64, 0)):
        assert size(*bad) == 0, bad
    p = [OK + i * BIG for i in range(16)]
    good = dict(dtype=1, x=p[0], M=10, D=64, wg=p[1], wu=p[2], F=128, wd=p[3], O=72, act=0, gate=p[4], up=p[5], y=p[6], ws=p[7],
                bytes=1 << 34)

    def call(**kw):
        return lib.pctc_gated_ffn(*dict(good, **kw).values(), None)

    assert call(M=0) == 0
    for bad in (dict(dtype=2), dict(M=-1), dict(D=60), dict(F=4), dict(O=0), dict(act=2), dict(gate=None), dict(up=None),
                dict(x=None), dict(wg=None), dict(wu=None), dict(wd=None), dict(y=None), dict(x=p[0] + 8), dict(wd=p[3] + 2),
                dict(gate=p[4] + 8), dict(y=p[0]), dict(gate=p[1] + 16), dict(up=p[4]), dict(y=p[5] + 16), dict(ws=p[7] + 8)):
        assert call(**bad) == -1, bad
    assert call(ws=None) == call(bytes=100) == -4
    good = dict(dtype=1, dy=p[0], x=p[1], M=10, D=64, gate=p[2], up=p[3], wg=p[4], wu=p[5], F=128, wd=p[6], O=72, act=1, dx=p[7],
                dwg=p[8], dwu=p[9], dwd=p[10], ws=p[11], bytes=1 << 34)

    def back(**kw):
        return lib.pctc_gated_ffn_backward(*dict(good, **kw).values(), None)

    for bad in (dict(dtype=2), dict(M=-1), dict(D=60), dict(F=4), dict(O=0), dict(act=-1), dict(dwg=None), dict(dwu=None),
                dict(dy=None), dict(x=None), dict(gate=None), dict(up=None), dict(wg=None), dict(wu=None), dict(wd=None),
                dict(dx=p[7] + 8), dict(dx=p[1]), dict(dwg=p[4]), dict(dwg=p[9]), dict(dwd=p[8] + 256), dict(ws=p[11] + 16)):
        assert back(**bad) == -1, bad
    assert back(ws=None) == back(bytes=100) == -4


@built
def test_entry_points_check_their_tensors():
    """The binding's own checks, on host tensors (nothing reaches the library)."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    x, w, t = torch.zeros(4, 8), torch.zeros(16, 8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: pc.dropout(x, 0.1, 1), lambda: pc.embedding(w, t), lambda: pc.embedding_backward(x, t, 16),
                 lambda: pc.gated_ffn(x, w, w, w.T), lambda: pc.gated_ffn_backward(x, x, x, x, w, w, w.T),
                 lambda: pc.gated_ffn(x, w, w, w.T, "relu"), lambda: pc.policy_loss(x, w, t, x[:, 0]),
                 lambda: pc.dropout(x.half(), 0.1, 1)):
        with pytest.raises(pc.PrunedCTCError):
            call()


@built
def test_a_workspace_that_meets_another_buffer_is_refused():
    """It is written: over an input it would change what the call reads, over an output what it gives."""
    lib = _lib()
    p = [OK + i * BIG for i in range(17)]
    room = 1 << 34
    # (name, arguments of which pointers may be any, the workspace's place, its size)
    calls = {
        "embedding_backward": (lib.pctc_embedding_backward, [1, p[0], p[1], 4, 50, 10, 8, 1.0, 0, p[2], 0, p[16], room, None], 11,
                               lib.pctc_embedding_backward_workspace_size(50, 8)),
        "gated_ffn": (lib.pctc_gated_ffn, [1, p[0], 10, 64, p[1], p[2], 128, p[3], 72, 0, p[4], p[5], p[6], p[16], room, None], 13,
                      lib.pctc_gated_ffn_workspace_size(1, 10, 64, 128, 72, 0)),
        "gated_ffn_backward": (lib.pctc_gated_ffn_backward, [1, p[0], p[1], 10, 64, p[2], p[3], p[4], p[5], 128, p[6], 72, 1, p[7],
                                                             p[8], p[9], p[10], p[16], room, None], 17,
                               lib.pctc_gated_ffn_workspace_size(1, 10, 64, 128, 72, 1)),
        "policy_loss": (lib.pctc_policy_loss, [1, p[0], 10, 64, p[1], p[2], 300, p[3], p[4], p[5], p[6], p[7], 0.2, 0.2, 0.1, 0,
                                               p[8], p[9], p[10], p[11], p[12], p[13], p[14], p[16], room, None], 23,
                        lib.pctc_policy_workspace_size(1, 10, 64, 300, 1, 1, 0)),
    }
    for name, (f, args, at, need) in calls.items():
        assert need > 0
        for q in [a for a in args if isinstance(a, int) and a >= OK and a != p[16]]:
            for ws in (q, q - (need - 1) // 256 * 256):  # at its start, and ending behind it
                args[at] = ws
                assert f(*args) == -1, (name, p.index(q), ws - q)
