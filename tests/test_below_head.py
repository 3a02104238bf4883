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
    assert size(100, 64) > 0 and size(20_000, 64) > size(16_000, 64)
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
