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


def rest_of(w, at):
    """1 - p and ln p of the word at `at`, from all weights relative to its own."""
    rows = np.arange(len(at))
    others = w.copy()
    others[rows, at] = 0.0
    x = others.sum(axis=1)
    return x / (1 + x), -np.log1p(x)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [60, 1_000, 33_278, 140_001])
@pytest.mark.parametrize("T,ws,wl", [(1.0, 0.0, 1.0), (1.0, 1.0, 0.0), (2.0, 0.6, 0.4), (3.0, 0.6, 0.4), (0.5, 0.6, 0.4), (2.0, 0.0, 1.0)])
def test_distillation_of_certain_words(rgc, ctx, dtype, vocab, T, ws, wl):      # noqa: F811
    """Label, the student's favourite and the teacher's are one word, and both are nearly certain of it: loss and gradient there are made of
    the rest's weights.  The loss' tolerance is relative to its terms' sizes, the gradient's at the word to 1 - p and 1 - q, elsewhere to p and q."""
    import torch
    g = np.random.default_rng(vocab + 1)
    z, at = certain_rows(g, vocab, T)
    n, k = len(at), 6
    rows = np.arange(n)
    index = np.stack([np.concatenate([[a], (a + 1 + g.permutation(vocab - 1)[:k - 1]) % vocab]) for a in at])
    teacher = g.standard_normal((n, k)).astype(np.float32)
    wanted = 10.0 ** g.uniform(-8, -3, n)
    teacher[:, 0] = T * np.log(np.exp(teacher[:, 1:].astype(np.float64) / T).sum(axis=1) / wanted)
    index[3, 4] = at[3]                                    # the word twice, as two halves
    teacher[3, 4] = teacher[3, 0]
    put = lambda v, kind: torch.tensor(v, dtype=kind, device="cuda")   # noqa: E731
    logits = plain.upload(z, dtype)
    loss, grad = torch.full((n,), 5.0, device="cuda"), torch.full_like(logits, 5.0)
    targets = put(at, torch.int32)
    rgc.rgc_distill_loss(ctx, rgc.Distillation(logits, put(index, torch.int32), put(teacher, torch.float32), targets=targets, loss=loss, grad_logits=grad,
                                               temperature=T, soft_weight=ws, label_weight=wl))
    logprob = torch.full((n,), 5.0, device="cuda")
    rgc.rgc_token_logprobs(ctx, rgc.TokenScores(logits, targets, logprob=logprob))
    torch.cuda.synchronize()
    used, t64 = plain.as64(logits), teacher.astype(np.float64)
    tol = 2 * plain.rel(vocab, 64) + 16 * plain.U
    d = used - used[rows, at][:, None]
    rest_p, log_p = rest_of(np.exp(d / T), at)
    rest_p1, log_p1 = rest_of(np.exp(d), at)
    logp, logp1 = d / T + log_p[:, None], d + log_p1[:, None]
    # the teacher's entries by word; the certain word's are one (at temperature T, relative to it)
    wt = np.zeros((n, vocab))
    for r in range(n):
        np.add.at(wt[r], index[r], np.exp((t64[r] - t64[r, 0]) / T))
    wt /= wt[rows, at][:, None]
    rest_q, log_q = rest_of(wt, at)
    q = wt * np.exp(log_q)[:, None]
    with np.errstate(all="ignore"):
        logq = np.log(wt) + log_q[:, None]
        terms = np.where(q > 0, q * (logq - logp), 0.0)
        sizes = np.where(q > 0, q * (np.abs(logq) + np.abs(logp) + 1), 0.0)
    sizes[rows, at] = (np.abs(log_q) + np.abs(log_p))
    want = ws * T * T * terms.sum(axis=1) - wl * log_p1
    slack = (ws * T * T * sizes.sum(axis=1) + wl * np.abs(log_p1)) * tol + 2.0 ** -126
    got = plain.as64(loss)
    assert (np.abs(got - want) <= slack).all(), (got, want, slack)
    if ws == 0.0:
        assert (np.abs(got + plain.as64(logprob)) <= 2 * slack).all()
    p, p1 = np.exp(logp), np.exp(logp1)
    want = ws * T * (p - q) + wl * p1
    size = ws * T * (p + q) + wl * p1
    want[rows, at] = ws * T * (rest_q - rest_p) - wl * rest_p1
    size[rows, at] = ws * T * (rest_q + rest_p) + wl * rest_p1
    off = np.abs(plain.as64(grad) - want)
    ok = off <= tol * size + 1.01 * plain.ROUNDING[dtype] * np.abs(want) + plain.SMALLEST[dtype]
    assert ok.all(), (np.argwhere(~ok)[:4], plain.as64(grad)[~ok][:4], want[~ok][:4])
