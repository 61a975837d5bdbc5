"""Loops of the language model's operators that go round more than once at sizes of their own: convolution gradients of more walks than the waves that share them, embedding gradients of more rows than
one round of the sort's prefix sums counts."""
import numpy as np
import pytest

from test_gpu_lm_convolution import check as check_convolution
from test_gpu_lm_embed import check as check_embedding, ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,steps,width,dtype", [(800, 3, 1_500, "f32"), (800, 3, 1_500, "bf16"), (350, 65, 1_500, "f16"), (2_100, 9, 500, "f32")])
def test_a_wave_takes_several_walks(rgc, ctx, batch, steps, width, dtype):      # noqa: F811
    """A walk is 64 steps of a sequence; for 128 channels there are at most 2048 / ceil(width / 128) + 1 workgroups, of four waves: 684 waves at width 1500, 2052 at 500."""
    walks, waves = batch * -(-steps // 64), 4 * (2_048 // -(-width // 128) + 1)
    assert walks > waves
    g = np.random.default_rng(batch)
    lengths = g.integers(0, min(steps, 8) + 1, batch)
    lengths[:: 50], lengths[1:: 77], lengths[-1] = steps, steps - 1, steps
    resets = (g.random((batch, steps)) < 0.2).astype(np.uint8)
    check_convolution(rgc, ctx, batch, steps, width, 4, dtype, lengths=lengths, resets=resets, garbage=True)


@pytest.mark.parametrize("rows,vocab", [(1_024 * 1_024 + 1, 300), (1_100_000, 70_000)])
@pytest.mark.parametrize("add", [False, True])
def test_a_million_rows(rgc, ctx, rows, vocab, add):      # noqa: F811
    """More than 1024 blocks of 1024 rows: a digit's counts are added up in two rounds."""
    g = np.random.default_rng(rows)
    tokens = g.integers(0, vocab, rows)
    tokens[g.random(rows) < 0.05] = -1
    check_embedding(rgc, ctx, tokens, vocab, 1, "bf16", "f32", 0.5, add=add)
