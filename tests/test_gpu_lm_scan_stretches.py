"""Scans of sequences that are cut into stretches of several chunks, as long prompts are: what a stretch tells the next is added up over chunks, whose rows of B and C lie in shared memory in turn.

The bounds are test_gpu_lm_scan.py's.  Its term for a stretch's decay, 80 u of the exponent for the sum of the sizes, is for sums of up to 80 numbers: here a lane adds up at most 64 one after the
other (one lane a channel has all of a stretch's, 2 chunks of 32; four lanes a quarter of 4 chunks, 32; eight an eighth of 3 chunks, 12; sixteen, two a step, an eighth of 2 chunks, 8), then the lanes'
sums on at most three levels (of the sixteen, half have none): 67 u.
How a call is cut is seen by the scratch that it needs: the forward call's is that of the stretches, 32-bit words [batch][stretches][width * (states + 1)] and one more each, in words of 64 bits."""
import numpy as np
import pytest

from test_gpu_lm_scan import check, ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu

CHUNK = 32
# batch, steps, width, states, groups, chunks of a stretch, stretches.  Few channels a group make many waves of little work: a wave has 64 of one state, 16 of up to 4 (these by one lane each), 8 of up
# to 16, 24 or 32, 4 of more.
SHAPES = {
    "one state": (7, 1_000, 100, 1, 100, 2, 16),
    "four states": (7, 1_000, 100, 4, 100, 2, 16),
    "sixteen states": (5, 2_230, 140, 16, 140, 4, 18),
    "twenty-four states": (7, 1_500, 100, 24, 100, 3, 16),
    "sixty-four states": (14, 1_000, 50, 64, 50, 2, 16),
}


def shape(name):
    batch, steps, width, states, groups, stretch, stretches = SHAPES[name]
    chunks = -(-steps // CHUNK)
    assert stretches == -(-chunks // stretch)
    return batch, steps, width, states, groups, stretch, stretches


def is_cut_into(rgc, batch, steps, width, states, groups, stretches, dtype="f32"):      # noqa: F811
    """Whether the forward call has so many stretches: it needs exactly their scratch."""
    import torch
    kind = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    zeros = lambda *s: torch.zeros(*s, dtype=kind, device="cuda")      # noqa: E731
    x, b = zeros(batch, steps, width), zeros(batch, steps, groups * states)
    call = rgc.Scan(x, x, torch.zeros(width, states, device="cuda"), b, b, torch.empty_like(x), groups=groups)
    words = (batch * stretches * (width * (states + 1) + 1) + 1) // 2
    status = []
    for have in (words - 1, words):
        c = rgc.Context(1024, 1)
        c.limit_optional_scratch(8 * have)
        try:
            rgc.rgc_selective_scan(c, call)
            status.append(0)
        except rgc.RgcError as e:
            status.append(e.status)
        torch.cuda.synchronize()
        c.close()
    return status == [-2, 0]


@pytest.mark.parametrize("name", list(SHAPES))
def test_the_cut(rgc, name):      # noqa: F811
    batch, steps, width, states, groups, _, stretches = shape(name)
    assert is_cut_into(rgc, batch, steps, width, states, groups, stretches)


def lengths_of(batch, steps, stretch):
    """Rows that end inside the first and the second chunk of a stretch, at its borders, in the last stretch, and nowhere."""
    s = CHUNK * stretch
    some = [steps, 0, steps - 1, CHUNK + 9, s, s + 5, s + CHUNK, s + CHUNK + 1, 2 * s - 1, steps - CHUNK, 1, s + 1, 3 * s + CHUNK - 1, steps - 2 * CHUNK - 3]
    return np.array(some[:batch], np.int32)


def resets_of(batch, steps, stretch):
    """Texts that begin inside the first and the second chunk of a stretch, at its borders, nowhere; a few anywhere."""
    s = CHUNK * stretch
    r = np.zeros((batch, steps), np.uint8)
    r[1] = np.random.default_rng(steps).random(steps) < 1.0 / 100.0
    r[2, [s, 2 * s]] = 1
    r[3, [s - 1, s + 1, 3 * s + CHUNK]] = 1
    r[4, [5, s + CHUNK + 3, steps - 1]] = 255
    return r


@pytest.mark.parametrize("name,dtype,layout", [("one state", "f32", "time"), ("four states", "bf16", "batch"), ("sixteen states", "f32", "batch"),
                                               ("twenty-four states", "f16", "slice"), ("sixty-four states", "bf16", "batch")])
@pytest.mark.parametrize("size", [0.02, 0.0005])
def test_whole_rows(rgc, ctx, name, dtype, layout, size):      # noqa: F811
    """Decays that are over within a stretch, and some that reach over several."""
    batch, steps, width, states, groups, _, _ = shape(name)
    check(rgc, ctx, batch, steps, width, states, groups, dtype, layout, train=False, size=size)


@pytest.mark.parametrize("name,dtype", [("one state", "bf16"), ("four states", "f32"), ("sixteen states", "bf16"), ("twenty-four states", "f32"), ("sixty-four states", "f32")])
def test_rows_that_end_and_texts_that_begin_inside_a_stretch(rgc, ctx, name, dtype):      # noqa: F811
    batch, steps, width, states, groups, stretch, _ = shape(name)
    lengths, resets = lengths_of(batch, steps, stretch), resets_of(batch, steps, stretch)
    check(rgc, ctx, batch, steps, width, states, groups, dtype, train=False, lengths=lengths, garbage=True, size=0.0005)
    check(rgc, ctx, batch, steps, width, states, groups, dtype, train=False, resets=resets, size=0.0005)
    check(rgc, ctx, batch, steps, width, states, groups, dtype, train=False, lengths=lengths, resets=resets, garbage=True, in_place=True)


@pytest.mark.parametrize("name", ["one state", "sixteen states"])
def test_training(rgc, ctx, name):      # noqa: F811
    """With the states that are kept for the backward pass, and the gradients made of them."""
    batch, steps, width, states, groups, stretch, _ = shape(name)
    check(rgc, ctx, batch, steps, width, states, groups, "f32", lengths=lengths_of(batch, steps, stretch), resets=resets_of(batch, steps, stretch), garbage=True, size=0.0005)


def test_several_waves_a_group(rgc, ctx):      # noqa: F811
    batch, steps, width, states, groups = 1, 1_000, 2_700, 16, 300                   # nine channels a group: two waves, the second with one
    assert is_cut_into(rgc, batch, steps, width, states, groups, 16, "bf16")
    check(rgc, ctx, batch, steps, width, states, groups, "bf16", train=False, size=0.0005)
