"""The selective scan's states and their gradients in place: h_last in the place of h0, dh0 in the place of dh_last."""
import numpy as np
import pytest

from test_gpu_lm_scan import check, ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("states", [1, 5, 16, 24, 64])
@pytest.mark.parametrize("steps", [0, 1, 35, 300])
def test_states_in_place(rgc, ctx, steps, states, dtype):      # noqa: F811
    """To the bounds of those that have a place of their own; the gradients are made of what the forward call kept, not of h0."""
    g = np.random.default_rng(steps)
    check(rgc, ctx, 3, steps, 37, states, dtype=dtype, in_place=True)
    check(rgc, ctx, 4, steps, 18, states, 2, dtype, "time", lengths=np.array([steps, 0, steps // 2, min(steps, 33)]), resets=(g.random((4, steps)) < 0.1).astype(np.uint8), garbage=True, in_place=True)


@pytest.mark.parametrize("states", [1, 5, 16, 24, 33, 64])
@pytest.mark.parametrize("steps", [0, 1, 20, 32, 33, 40, 48, 49, 200])
def test_gradients_of_states_in_place(rgc, ctx, steps, states):      # noqa: F811
    """One chunk, a sequence of a few steps more that is taken as one, several chunks; rows without steps, rows that end in the first chunk, widths that leave lanes behind a group's end.
    The same bits as with a place of its own."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(steps)
    batch, width, groups = 4, 46, 2
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    x, delta, gate, dy, b, c = (rand(batch, steps, n) for n in (width, width, width, width, groups * states, groups * states))
    a, h0, dh_last = -torch.rand(width, states, generator=g, device="cuda"), rand(batch, width, states), rand(batch, width, states)
    for lengths in (None, torch.tensor([steps, 0, steps // 2, min(steps, 7)], dtype=torch.int32, device="cuda")):
        call = rgc.Scan(x, delta, a, b, c, torch.empty_like(x), groups=groups, gate=gate, softplus=True, lengths=lengths, h0=h0,
                        states=torch.empty(batch, -(-steps // rgc.RGC_SCAN_CHUNK), width, states, device="cuda"))
        rgc.rgc_selective_scan(ctx, call)
        got = []
        for in_place in (False, True):
            known = dh_last.clone()
            out = {"dx": x, "ddelta": x, "dgate": x, "db": b, "dc": b, "da": a, "dh0": dh_last}
            out = {k: torch.full_like(v, 5.0) for k, v in out.items()}
            if in_place:
                out["dh0"] = known
            rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, dy, out["dx"], out["ddelta"], out["da"], out["db"], out["dc"], dgate=out["dgate"], dh_last=known, dh0=out["dh0"]))
            torch.cuda.synchronize()
            got.append(out)
        for k, v in got[0].items():
            assert torch.equal(v, got[1][k]), k
        if steps > 0 and lengths is not None:
            assert torch.equal(got[1]["dh0"][1], dh_last[1])           # a row without steps hands on what comes in
