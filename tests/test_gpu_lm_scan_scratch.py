"""How many workgroups the selective scan's backward call shares its channels among, seen by the scratch that it needs: a few hundred, whether rows have lengths or not; more only for rows of several
chunks that may end early, and none with fewer than eight stretches of a wave's channels."""
import pytest

from test_gpu_lm_scan import rgc      # noqa: F401  (fixture)

pytestmark = pytest.mark.gpu

CHUNK = 32


def bytes_of(batch, steps, width, states, groups, splits):
    chunks = 1 if steps <= 48 and states <= 32 else -(-steps // CHUNK)
    joined = batch * chunks if chunks > 1 else 0
    words = joined * (width * states + width + 1) + batch * chunks * width * (states + 2) + splits * batch * steps * 2 * groups * states
    return 8 * ((words + 1) // 2)


@pytest.mark.parametrize("batch,steps,width,states,groups,alone,with_lengths", [
    (20, 35, 1_500, 16, 1, 25, 25),                      # one chunk: 512 / 20, of 188 stretches of 8 channels
    (64, 16, 300, 16, 1, 8, 8),
    (3, 48, 100, 8, 1, 7, 7),                            # as many as there are stretches (of 16 channels)
    (2, 500, 768, 16, 1, 16, 16),                        # 512 / 32; 96 stretches are twelve times eight
    (6, 1_001, 1_502, 16, 1, 2, 10),                     # 512 / 192, and 2048 / 192
    (8, 100, 1_024, 16, 2, 8, 8),                        # 512 / 64; 2048 / 64, but 64 stretches a group
    (8, 200, 1_024, 32, 1, 9, 32),                       # 2048 / 56, but 256 stretches of 4 channels
    (300, 70, 40, 4, 1, 1, 1),
])
def test_scratch_of_the_backward_call(rgc, batch, steps, width, states, groups, alone, with_lengths):      # noqa: F811
    import torch
    zeros = lambda *s: torch.zeros(*s, device="cuda")      # noqa: E731
    x, b, a = zeros(batch, steps, width), zeros(batch, steps, groups * states), zeros(width, states)
    kept = zeros(batch, -(-steps // CHUNK), width, states)
    for lengths, splits in ((None, alone), (torch.full((batch,), steps, dtype=torch.int32, device="cuda"), with_lengths)):
        call = rgc.Scan(x, x, a, b, b, torch.empty_like(x), groups=groups, lengths=lengths, states=kept)
        grads = rgc.ScanGrads(call, x, torch.empty_like(x), torch.empty_like(x), torch.empty_like(a), torch.empty_like(b), torch.empty_like(b))
        status = []
        for have in (bytes_of(batch, steps, width, states, groups, splits) - 8, bytes_of(batch, steps, width, states, groups, splits)):
            ctx = rgc.Context(1024, 1)
            ctx.limit_optional_scratch(have)
            try:
                rgc.rgc_selective_scan_backward(ctx, call, grads)
                status.append(0)
            except rgc.RgcError as e:
                status.append(e.status)
            torch.cuda.synchronize()
            ctx.close()
        assert status == [-2, 0], (lengths is not None, status)
