"""A workgroup of a long recurrence that waits for words which do not come ends all the same.  The words are there at the first look or not, as it
happens, when it may look once only (rgc_limit_looks): every result is then the right one, bit for bit, or NaN, and with the library's own limit all
are right again."""
import pytest

from test_gpu_lm_recurrence import ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("looks", [1, 3])
@pytest.mark.parametrize("dtype,batch,steps,width", [("float32", 1, 50_000, 64), ("bfloat16", 2, 9_000, 700), ("float32", 3, 700, 200)])
def test_a_wait_that_is_given_up(rgc, ctx, dtype, batch, steps, width, looks):      # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(steps)
    kind = getattr(torch, dtype)
    x, gate, og, dy = (torch.randn(batch, steps, width, generator=g, device="cuda").to(kind) for _ in range(4))
    gate = gate + 4

    def both():
        out = {k: torch.empty_like(x) for k in ("y", "dx", "dgate", "dout_gate")}
        out.update(h_last=torch.empty(batch, width, device="cuda"), dh0=torch.empty(batch, width, device="cuda"),
                   states=torch.empty(batch, -(-steps // rgc.RGC_RECURRENCE_CHUNK), width, device="cuda"))
        call = rgc.Recurrence(x, gate, out["y"], out_gate=og, h_last=out["h_last"], states=out["states"])
        rgc.rgc_gated_recurrence(ctx, call)
        rgc.rgc_gated_recurrence_backward(ctx, call, rgc.RecurrenceGrads(call, dy, out["dx"], out["dgate"], dout_gate=out["dout_gate"], dh0=out["dh0"]))
        torch.cuda.synchronize()
        return out

    want = both()
    ctx.limit_looks(looks)
    try:
        for _ in range(3):
            got = both()
            for k in want:
                assert bool(((got[k] == want[k]) | got[k].isnan()).all()), k
    finally:
        ctx.limit_looks(-1)
    again = both()
    for k in want:
        assert torch.equal(want[k], again[k]), k


def test_refusals(rgc, ctx):      # noqa: F811
    with pytest.raises(rgc.RgcError) as e:
        ctx.limit_looks(0)
    assert e.value.status == -1
    assert rgc.load_library().rgc_limit_looks(None, 1) == -1
