"""Distillation where a teacher's index comes more than once: it stands for the sum of its entries' weights, in the loss as in the
gradient.  The oracle joins such entries into one, whose logit is T ln sum exp(logit / T), before the definition in 64 bits is
applied; the tolerances are those of the distillation's other tests, with the joined entries' weights in them."""
import numpy as np
import pytest

import test_gpu_lm_vocab as plain
from test_gpu_lm_vocab import ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def joined(index, teacher, T, vocab):
    """One entry for every index of a row; the places of the others are left out."""
    index, teacher = index.copy(), teacher.copy()
    for r in range(index.shape[0]):
        first = {}
        for i, at in enumerate(index[r]):
            if not 0 <= at < vocab:
                continue
            if at in first:
                with np.errstate(all="ignore"):
                    teacher[r, first[at]] = T * np.logaddexp(teacher[r, first[at]] / T, teacher[r, i] / T)
                index[r, i] = -1
            else:
                first[at] = i
    return index, teacher


@pytest.fixture(autouse=True)
def oracle_of_sums(monkeypatch):
    separate = plain.distill64

    def of_sums(z, index, teacher, targets, T, *rest):
        index, teacher = joined(index, teacher, T, z.shape[1])
        return separate(z, index, teacher, targets, T, *rest)

    monkeypatch.setattr(plain, "distill64", of_sums)


WEIGHTS = ((1.0, 1.0, 0.0), (2.0, 0.5, 0.5), (3.0, 0.7, 0.3), (1.0, 0.0, 1.0), (3.0, 0.0, 0.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab,k", [(40, 2), (3_000, 40), (10_000, 128), (140_001, 128)])
def test_an_index_that_comes_more_than_once(rgc, ctx, dtype, vocab, k):      # noqa: F811
    g = np.random.default_rng(vocab + k)
    z = plain.logits_like(g, 6, vocab)
    index, teacher = plain.teacher_like(g, z, k)
    index[0, k // 2:] = index[0, :k - k // 2]          # every index twice
    index[1] = index[1, 0]                             # one index alone
    index[2] = index[2, g.integers(0, max(1, k // 8), k)]     # some many times
    index[3, -1] = index[3, 0]                         # one twice, as far apart as they can be
    index[4, 1] = index[4, 0]
    teacher[4, 1] = -np.inf                            # ... the second without weight
    targets = g.integers(0, vocab, 6)
    targets[[1, 2]] = index[[1, 2], 0]
    for T, ws, wl in WEIGHTS:
        plain.check_distill(rgc, ctx, z, index, teacher, targets, dtype, T, ws, wl)
        plain.check_distill(rgc, ctx, z, index, teacher, None, dtype, T, ws, wl)


def test_entries_left_out_twice_and_masked(rgc, ctx):      # noqa: F811
    g = np.random.default_rng(21)
    vocab, k = 3_000, 40
    z = plain.logits_like(g, 12, vocab)
    index, teacher = plain.teacher_like(g, z, k)
    index[1, 5:] = -1                                  # fewer entries
    teacher[1, 5:] = np.nan                            # what lies in their place is not looked at
    index[2] = vocab                                   # no entry at all
    index[3, 20:] = index[3, :20]                      # entries that come twice
    teacher[4] = -np.inf                               # entries without weight
    teacher[5, 3:] = -np.inf
    index[6] = -1
    z[6] = np.nan                                      # a row with neither teacher nor label
    z[7] = -np.inf
    z[8, index[8]] = -np.inf                           # the student rules out all that the teacher wants
    teacher[9, 0] = np.nan
    teacher[10] = -3.4028234e38
    teacher[11, 0] = 3.0e38
    targets = g.integers(0, vocab, 12)
    targets[[2, 6]] = -1
    targets[3] = index[3, 0]
    for dtype in ("f32", "bf16"):
        for T, ws, wl in WEIGHTS:
            plain.check_distill(rgc, ctx, z, index, teacher, targets, dtype, T, ws, wl)
            plain.check_distill(rgc, ctx, z, index, teacher, None, dtype, T, ws, wl)


@pytest.mark.parametrize("vocab", [1_000, 140_001])
def test_a_student_that_agrees_has_no_loss(rgc, ctx, vocab):      # noqa: F811
    """All of the teacher's weight on one word, in two halves, and a student that is certain of it: the divergence is 0."""
    import torch
    z = torch.full((2, vocab), -60.0, device="cuda")
    z[:, 3] = 60.0
    index = torch.full((2, 2), 3, dtype=torch.int32, device="cuda")
    loss, grad = torch.full((2,), 5.0, device="cuda"), torch.full_like(z, 5.0)
    rgc.rgc_distill_loss(ctx, rgc.Distillation(z, index, torch.zeros(2, 2, device="cuda"), loss=loss, grad_logits=grad))
    torch.cuda.synchronize()
    # ln q and ln p carry a rounding of fp32's 2 and 1 each, their difference nothing else
    assert float(loss.abs().max()) <= 4 * plain.U and float(grad.abs().max()) <= 4 * plain.U
