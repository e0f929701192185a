"""Ends of the ranges that the header promises for log probabilities: the signs of log probabilities and entropies.

Tolerances are derived, not measured.  A rounding is off by half a step (relative 2^-24 in fp32, 2^-8 in bf16)."""
import numpy as np
import pytest

import test_gpu_more_operators as G
from paper_2203_12533_amd import binding as pwb

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    with pwb.Context(0) as c:
        yield c


# ---- log probabilities: signs ----------------------------------------------------------------------------------

@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("rows,vocab,scale", [(600, 1, 1.0), (600, 2, 0.7), (600, 130, 1.0), (200, 3000, 1.3), (600, 9000, 1.0), (40, 40000, 1.0),
                                              (40, 40000, 37.0)])
def test_log_probabilities_are_at_most_zero_and_entropies_at_least(ctx, rows, vocab, scale, bf16):
    """Rows with one token that is nearly certain, its logit of any size: the sum of the others is at, far below and above a rounding of
    1.  A NaN in a row still shows."""
    rng = np.random.RandomState(vocab)
    top = rng.uniform(1, 100, rows) * np.where(np.arange(rows) % 2, 1, -1) * 10.0 ** rng.randint(-2, 4, rows)
    z = top[:, None] - (rng.uniform(8, 30, (rows, 1)) + rng.rand(rows, vocab)) / scale
    t = rng.randint(0, vocab, rows)
    z[np.arange(rows), t] = top
    z[7, 0] = np.nan
    k = min(3, vocab)
    lp, en, st, ids, tl = G.logprob(ctx, z, t, scale, k, bf16, backward=False)
    lp, en, st, tl = G.back(lp)[0, :rows], G.back(en)[0, :rows], G.back(st), G.back(tl)
    ok = np.arange(rows) != 7
    assert (lp[ok] <= 0).all() and (tl[ok] <= 0).all(), (lp[ok].max(), tl[ok].max())
    assert (en[ok] >= 0).all() and (st[ok, 1] >= 0).all(), (en[ok].min(), st[ok, 1].min())
    assert np.isnan(lp[7]) and np.isnan(en[7]) and np.isnan(tl[7]).all() and np.isnan(st[7, 1])
