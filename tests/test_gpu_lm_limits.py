"""Operators over rows of logits at the ends of their ranges: the largest vocabulary (64 segments, and 128 entries of each to merge), gradients in
the place of the logits, and gradients without targets."""
import math

import numpy as np
import pytest

import test_gpu_lm_vocab as plain
from test_gpu_lm_vocab import ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

VOCAB_MAX = 4_194_304


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,top", [(1, VOCAB_MAX, 128), (2, VOCAB_MAX - 1, 5), (1, 1_048_577, 128), (130, 65_537, 20), (130, 131_073, 7)])
def test_scores_of_the_longest_rows(rgc, ctx, dtype, rows, vocab, top):      # noqa: F811
    g = np.random.default_rng(vocab)
    z = plain.logits_like(g, rows, vocab)
    z[0, ::vocab // 300] += 9.0                              # the alternatives come from all segments
    targets = g.integers(0, vocab, rows)
    targets[0] = vocab - 1
    grads = (g.standard_normal(rows), g.standard_normal(rows))
    used, got = plain.run_scores(rgc, ctx, z, dtype, targets, top, 1.0, grads=grads)
    some = np.unique(np.concatenate([[0, rows - 1], g.integers(0, rows, 3)]))
    got = {k: v[some] for k, v in got.items()}
    plain.check_scores(used[some], got, targets[some], dtype, top, 1.0, tuple(v[some] for v in grads))


def test_more_words_than_the_largest_vocabulary(rgc, ctx):      # noqa: F811
    import torch
    z = torch.zeros(1, VOCAB_MAX + 1, device="cuda")
    f, idx, val = torch.zeros(1, device="cuda"), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, device="cuda")
    for call in (lambda: rgc.rgc_token_logprobs(ctx, rgc.TokenScores(z, entropy=f)), lambda: rgc.rgc_distill_loss(ctx, rgc.Distillation(z, idx, val, loss=f))):
        with pytest.raises(rgc.RgcError) as e:
            call()
        assert e.value.status == -1


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 1), (5, 3), (64, 7)])
@pytest.mark.parametrize("vocab", [13, 1_000, 33_278])
def test_gradient_in_the_place_of_the_logits(rgc, ctx, dtype, pad, shift, vocab):      # noqa: F811
    """It is the gradient that a tensor of its own gets, and what lies between the rows is not touched."""
    import torch
    g = np.random.default_rng(pad * 100 + shift + vocab)
    z = plain.logits_like(g, 6, vocab)
    targets = np.array([0, vocab - 1, vocab // 2, -1, vocab, 3])
    weight, bonus = (torch.tensor(g.standard_normal(6), dtype=torch.float32, device="cuda") for _ in range(2))
    for grads in ((weight, None), (None, bonus), (weight, bonus)):
        logits = plain.upload(z, dtype, pad, shift)
        out = {"logprob": torch.empty(6, device="cuda"), "entropy": torch.empty(6, device="cuda"), "stats": torch.empty(6, 2, device="cuda")}
        call = rgc.TokenScores(logits, torch.tensor(targets, dtype=torch.int32, device="cuda"), temperature=2.0, **out)
        rgc.rgc_token_logprobs(ctx, call)
        used, beside = plain.as64(logits), torch.full((6, vocab + 2), 55.0, dtype=logits.dtype, device="cuda")
        rgc.rgc_token_logprobs_backward(ctx, call, beside[:, :vocab], *grads)
        rgc.rgc_token_logprobs_backward(ctx, call, logits, *grads)
        torch.cuda.synchronize()
        got = {k: plain.as64(v) for k, v in out.items()}
        got["grad"] = plain.as64(logits)
        plain.check_scores(used, got, targets, dtype, 0, 2.0, tuple(None if v is None else plain.as64(v) for v in grads))
        assert torch.equal(beside[:, :vocab], logits) and bool((beside[:, vocab:] == 55.0).all())
        whole = logits.as_strided((6 * (vocab + pad) + shift,), (1,), 0)
        assert bool(whole[:shift].isnan().all()) and bool(whole[shift:].view(6, vocab + pad)[:, vocab:].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [50, 2_000, 70_001])
def test_gradient_without_targets(rgc, ctx, dtype, vocab):      # noqa: F811
    g = np.random.default_rng(vocab)
    z = plain.logits_like(g, 4, vocab)
    z[1, ::2] = -math.inf
    z[2] = -math.inf
    grads = (None, g.standard_normal(4))
    used, got = plain.run_scores(rgc, ctx, z, dtype, None, 6, 0.5, grads=grads)
    plain.check_scores(used, got, None, dtype, 6, 0.5, grads)
    assert np.all(got["grad"][2] == 0) and np.any(got["grad"][0] != 0)


def test_gradient_in_the_logits_place_with_other_rows_is_refused(rgc, ctx):      # noqa: F811
    """Its rows would lie over other rows' logits."""
    import torch
    flat = torch.zeros(4 * 16, device="cuda")
    logits, closer = flat.view(4, 16)[:, :10], flat.as_strided((4, 10), (10, 1))
    t, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    scores = rgc.TokenScores(logits, t, logprob=f, stats=torch.zeros(4, 2, device="cuda"))
    idx, val = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda")
    for call in (lambda: rgc.rgc_token_logprobs_backward(ctx, scores, closer, f),
                 lambda: rgc.rgc_distill_loss(ctx, rgc.Distillation(logits, idx, val, grad_logits=closer)),
                 lambda: rgc.rgc_distill_loss(ctx, rgc.Distillation(closer, idx, val, grad_logits=logits))):
        with pytest.raises(rgc.RgcError) as e:
            call()
        assert e.value.status == -1
    # one row has no stride
    rgc.rgc_distill_loss(ctx, rgc.Distillation(logits[:1], idx[:1], val[:1], grad_logits=closer[:1]))
    torch.cuda.synchronize()
