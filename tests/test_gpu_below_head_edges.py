"""Calls of dropout, token embedding, the gated block and the policy loss at the edges of what they take, on the GPU
(through the public binding), against 64-bit references or exact values."""
import math

import numpy as np
import pytest

from tests import below_head_ref as ref
from tests.gpu_util import say
from tests.test_gpu_below_head import check_ffn, check_grad, check_policy, dev, ffn_case, host, kind, policy_call, policy_case

pytestmark = pytest.mark.gpu


# ---- values that change lanes ------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,D,F_", [(300, 64, 8328), (520, 72, 776), (90, 520, 264)])
def test_gated_ffn_projections_of_whole_numbers(dtype, M, D, F_):
    """Sums of whole numbers are exact in any order: a value that a lane took from another place of its exchange
    would differ by whole numbers."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("gated_ffn whole numbers", dtype, M, D, F_)
    r = np.random.default_rng(M)
    x, wg, wu = (r.integers(-3, 4, size=s).astype(np.float32) for s in ((M, D), (F_, D), (F_, D)))
    got = pc.gated_ffn(dev(x, dtype), dev(wg, dtype), dev(wu, dtype), torch.zeros(8, F_, device="cuda").to(kind(dtype)), keep=True)
    for k, w in (("gate", wg), ("up", wu)):
        assert np.array_equal(host(got[k]), x.astype(np.float64) @ w.T.astype(np.float64)), k


@pytest.mark.parametrize("N,V", [(15_361, 40), (20_000, 1100), (70_000, 524_288)])
def test_embedding_backward_of_whole_numbers(N, V):
    """The same of the sort: 64 places at a time with one digit, with many and with one token each."""
    import torch
    from paper_2609_33645_amd import prunedctc as pc
    say("embedding_backward whole numbers", N, V)
    r = np.random.default_rng(N)
    place = np.arange(N)
    for t in (place % V, np.where(place // 64 % 2 == 0, 3, place % V), r.integers(-1, V + 1, size=N)):
        dy = r.integers(-8, 9, size=(N, 3)).astype(np.float32)
        want = np.zeros((V, 3))
        ok = (t >= 0) & (t < V)
        np.add.at(want, t[ok], dy[ok].astype(np.float64))
        got = pc.embedding_backward(dev(dy), torch.from_numpy(t).cuda(), V)
        assert np.array_equal(host(got), want)
