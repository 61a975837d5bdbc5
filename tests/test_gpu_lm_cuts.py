"""Distillation at the lengths where rows are cut otherwise, up to the largest vocabulary: every way of cutting has a kernel, and loss and gradient are
those of the definition."""
import numpy as np
import pytest

import test_gpu_lm_vocab as plain
from test_gpu_lm_vocab import ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

VOCAB_MAX = 4_194_304


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,k,T", [(1, VOCAB_MAX, 128, 2.0), (1, VOCAB_MAX - 3, 3, 1.0), (1, 1_048_577, 128, 3.0), (130, 65_537, 20, 2.0), (130, 131_073, 20, 1.0),
                                            (2, 16_385, 9, 2.0), (2, 32_769, 9, 2.0), (127, 16_391, 9, 1.0), (129, 32_771, 9, 2.0)])
def test_distillation_of_the_longest_rows_and_at_the_cuts(rgc, ctx, dtype, rows, vocab, k, T):      # noqa: F811
    g = np.random.default_rng(vocab + k)
    z = plain.logits_like(g, rows, vocab)
    z[0, ::max(1, vocab // 300)] += 9.0
    index, teacher = np.empty((rows, k), np.int64), np.empty((rows, k), np.float32)
    for r in range(rows):
        index[r] = np.argpartition(-z[r], k)[:k]
        teacher[r] = z[r, index[r]] + g.standard_normal(k)
    index[0, 0], targets = vocab - 1, g.integers(0, vocab, rows)
    plain.check_distill(rgc, ctx, z, index, teacher, targets, dtype, T, 0.6, 0.4)
