"""The short convolution's gradients where the forward call put the kept inputs `last` in the place of `before`: what it read is gone then, and the backward call needs it."""
import pytest

from test_gpu_lm_convolution import check, ctx, rgc      # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


def tensors(dtype, batch=3, steps=1, width=70, taps=4):
    import torch
    g = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    return {"x": rand(batch, steps, width).to(dtype), "weight": rand(width, taps), "before": rand(batch, taps - 1, width).to(dtype), "dy": rand(batch, steps, width).to(dtype),
            "dlast": rand(batch, taps - 1, width).to(dtype)}


def outputs(t):
    import torch
    five = lambda like: torch.full_like(like, 5.0)      # noqa: E731
    return {"dx": five(t["x"]), "dweight": five(t["weight"]), "dbefore": five(t["before"])}


def backward(rgc, ctx, t, call):      # noqa: F811
    import torch
    out = outputs(t)
    status = 0
    try:
        rgc.rgc_causal_convolution_backward(ctx, call, rgc.ConvolutionGrads(call, t["dy"], out["dx"], out["dweight"], dlast=t["dlast"], dbefore=out["dbefore"]))
    except rgc.RgcError as e:
        status = e.status
    torch.cuda.synchronize()
    return status, out


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("taps", [2, 4, 8])
def test_a_backward_call_over_replaced_inputs_is_refused(rgc, ctx, taps, silu):      # noqa: F811
    import torch
    t = tensors(torch.float32, taps=taps)
    y, apart = torch.empty_like(t["x"]), torch.empty_like(t["before"])
    call = rgc.Convolution(t["x"], t["weight"], y, silu=silu, before=t["before"], last=apart)
    rgc.rgc_causal_convolution(ctx, call)
    status, want = backward(rgc, ctx, t, call)
    assert status == 0
    # the serving form: the call itself is right, its gradients are refused, and nothing is written
    kept, y_in = t["before"].clone(), torch.empty_like(y)
    in_place = rgc.Convolution(t["x"], t["weight"], y_in, silu=silu, before=kept, last=kept)
    rgc.rgc_causal_convolution(ctx, in_place)
    torch.cuda.synchronize()
    assert torch.equal(y_in, y) and torch.equal(kept, apart)
    status, got = backward(rgc, ctx, t, in_place)
    assert status == -1 and all(bool((v == 5.0).all()) for v in got.values())
    # with the inputs that it read, kept elsewhere, they are what they were
    status, got = backward(rgc, ctx, t, rgc.Convolution(t["x"], t["weight"], y_in, silu=silu, before=t["before"]))
    assert status == 0
    for k in want:
        assert torch.equal(got[k], want[k]), k


def test_where_nothing_is_replaced_it_is_not_refused(rgc, ctx):      # noqa: F811
    check(rgc, ctx, 3, 0, 9, 4, "bf16", in_place=True)                 # no steps: the kept inputs are handed on
    check(rgc, ctx, 0, 1, 9, 4, "f32", in_place=True)
    check(rgc, ctx, 3, 1, 9, 1, "f32", in_place=True)                  # one tap keeps none
    check(rgc, ctx, 3, 5, 9, 1, "f16", in_place=True)
    check(rgc, ctx, 3, 1, 301, 4, "bf16", in_place=True, train=False)
