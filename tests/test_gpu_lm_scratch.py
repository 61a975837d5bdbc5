"""Scratch of the language model's operators where the device is short of memory (rgc_limit_optional_scratch stands for that): a call gets what
it needs where twice the last buffer is not to be had, and one that needs more is refused and does nothing."""
import pytest

from test_gpu_lm_recurrence import rgc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

STEPS, WIDTH = 300, 64                         # three tiles of a chain of 64 channels: 3 * 64 words of 8 bytes a sequence


def bytes_of(batch):
    return 8 * (batch * 3 * 64 + 1)


def run(rgc, ctx, batch):      # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(batch)
    x, gate = (torch.randn(batch, STEPS, WIDTH, generator=g, device="cuda") for _ in range(2))
    y = torch.full_like(x, 5.0)
    try:
        rgc.rgc_gated_recurrence(ctx, rgc.Recurrence(x, gate, y))
        status = 0
    except rgc.RgcError as e:
        status = e.status
    torch.cuda.synchronize()
    return status, y


def test_what_is_needed_where_twice_as_much_is_not_there(rgc):      # noqa: F811
    plenty, short = rgc.Context(1024, 1), rgc.Context(1024, 1)
    try:
        assert run(rgc, short, 100)[0] == 0
        short.limit_optional_scratch(bytes_of(150))
        for batch in (120, 150):                                 # twice what it has is more than the cap
            status, y = run(rgc, short, batch)
            assert status == 0 and bool((y == run(rgc, plenty, batch)[1]).all())
        status, y = run(rgc, short, 151)
        assert status == -2 and bool((y == 5.0).all())
        assert run(rgc, short, 150)[0] == 0                      # what there is serves on
        short.limit_optional_scratch(-1)
        status, y = run(rgc, short, 151)
        assert status == 0 and bool((y == run(rgc, plenty, 151)[1]).all())
    finally:
        plenty.close()
        short.close()
