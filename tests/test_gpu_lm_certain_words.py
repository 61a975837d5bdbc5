"""Rows with one word that is certain but for x = 1e-9 .. 1e-4 of the others' weight: what is made of 1 - p keeps fp32's relative precision.

Tolerances.  x is a sum of the other weights, with the relative error rel(n, a) of such sums (test_gpu_lm_vocab.py; a: the exponents' size in
powers of two, below 64 here); log1p and expm1 add a few units in the last place each, 16 u together; everything is relative to
1 - p and to the entropy, which is made of the same x.  The result is rounded to its type once."""
import numpy as np
import pytest

import test_gpu_lm_vocab as plain
from test_gpu_lm_vocab import ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def certain_rows(g, vocab, T):
    """Rows whose favourite leaves the others a weight between 1e-9 and 1e-4, and where it is."""
    wanted = np.array([1e-9, 1e-8, 2e-8, 1e-7, 2e-7, 1e-6, 1e-5, 1e-4])
    z = 0.25 * g.standard_normal((len(wanted), vocab))
    at = g.integers(0, vocab, len(wanted))
    at[:2] = 0, vocab - 1
    rows = np.arange(len(wanted))
    z[rows, at] = -np.inf
    others = np.exp(z / T).sum(axis=1)
    z[rows, at] = T * np.log(others / wanted)
    return z.astype(np.float32), at


def exactly(used, at, T):
    """1 - p, ln p and the entropy of the certain word's row, without a difference of near numbers."""
    rows = np.arange(len(at))
    d = (used - used[rows, at][:, None]) / T
    w = np.exp(d)
    w[rows, at] = 0.0
    x = w.sum(axis=1)
    logp = -np.log1p(x)
    with np.errstate(all="ignore"):
        spread = np.where(w > 0, w * (d + logp[:, None]), 0.0).sum(axis=1)
    return x, x / (1 + x), logp, -spread / (1 + x) - logp / (1 + x)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("vocab", [7, 1_000, 33_278, 140_001])
@pytest.mark.parametrize("T", [1.0, 0.5, 3.0])
def test_gradient_at_a_certain_target(rgc, ctx, dtype, vocab, T):      # noqa: F811
    g = np.random.default_rng(vocab)
    z, at = certain_rows(g, vocab, T)
    rows = np.arange(len(at))
    tol = 2 * plain.rel(vocab, 64) + 16 * plain.U
    for grads in ((g.standard_normal(len(at)), None), (None, g.standard_normal(len(at))), (g.standard_normal(len(at)), 0.1 * g.standard_normal(len(at)))):
        used, got = plain.run_scores(rgc, ctx, z, dtype, at, 0, T, grads=grads)
        x, rest, logp, entropy = exactly(used, at, T)
        assert (x < 1e-3).all()
        gr, hr = (np.zeros(len(at)) if v is None else v.astype(np.float32).astype(np.float64) for v in grads)
        want = (gr * rest - hr * (1 - rest) * (logp + entropy)) / T
        size = (np.abs(gr) * rest + np.abs(hr) * (entropy + np.abs(logp))) / T
        off = np.abs(got["grad"][rows, at] - want)
        slack = tol * size + 1.01 * plain.ROUNDING[dtype] * np.abs(want) + plain.SMALLEST[dtype]
        assert (off <= slack).all(), (got["grad"][rows, at], want)
        if dtype == "f32" and grads[1] is None:
            # a row's gradient adds up to nothing (each entry rounded once, the sum of the others as large as the target's)
            assert (np.abs(got["grad"].sum(axis=1)) <= 2 * slack).all()
