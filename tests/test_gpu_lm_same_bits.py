"""Long recurrences give the same bits every time: which of a chain's tiles had published their states when a later one looked is a matter
of time, and must not be seen in a result.  Gates near 7.5 keep a state over thousands of steps, so that every tile's words count; the
calls run alone, behind each other, and beside other work, which moves the tiles against each other."""
import pytest

from test_gpu_lm_recurrence import ctx, dtype_of, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,batch,steps,width,slope", [("f32", 1, 20_000, 1_000, 7.5), ("bf16", 1, 20_000, 1_500, 7.5), ("f32", 6, 3_000, 700, 7.0),
                                                           ("bf16", 2, 6_000, 2_048, 4.0), ("f32", 1, 50_000, 64, 8.0)])
def test_repeated_calls_of_long_sequences(rgc, ctx, dtype, batch, steps, width, slope):      # noqa: F811
    import torch
    g = torch.Generator(device="cuda").manual_seed(steps + width)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    kind = dtype_of(dtype)
    x, og, dy = (normal(batch, steps, width).to(kind) for _ in range(3))
    gate = (slope + 0.3 * normal(batch, steps, width)).to(kind)
    h0, last = normal(batch, width), normal(batch, width)

    def one():
        out = {k: torch.empty_like(x) for k in ("y", "dx", "dgate", "dout_gate")}
        out.update(h_last=torch.empty(batch, width, device="cuda"), dh0=torch.empty(batch, width, device="cuda"),
                   states=torch.empty(batch, -(-steps // rgc.RGC_RECURRENCE_CHUNK), width, device="cuda"))
        call = rgc.Recurrence(x, gate, out["y"], out_gate=og, h0=h0, h_last=out["h_last"], states=out["states"])
        grads = rgc.RecurrenceGrads(call, dy, out["dx"], out["dgate"], dout_gate=out["dout_gate"], dh_last=last, dh0=out["dh0"])
        stream = torch.cuda.current_stream()
        rgc.rgc_gated_recurrence(ctx, call, stream)
        rgc.rgc_gated_recurrence_backward(ctx, call, grads, stream)
        return out

    first = one()
    torch.cuda.synchronize()
    side, busy = torch.cuda.Stream(), torch.zeros(1 << 26, device="cuda")
    torch.cuda.synchronize()
    for i in range(16):
        if i % 4 == 3:
            with torch.cuda.stream(side):
                for _ in range(4):
                    busy += 1.0
        again = one()
        if i % 2:
            torch.cuda.synchronize()
        for k in first:
            assert torch.equal(first[k], again[k]), "%s, call %d: %d bits of results differ" % (k, i, int((first[k] != again[k]).sum()))
    torch.cuda.synchronize()
