"""The short causal convolution and its gradients against the definition in 64 bits, input by input.

Tolerances.  u = 2^-24.  s is a sum of K + 1 numbers, made by K fused steps: off by at most K u A, A = |bias| + sum |w u|.  A sigmoid's exponent is off by (1.5 |s|) u relative, its power and
reciprocal by 2 u each: open and 1 - open by (1.5 |s| + 6) u relative, so silu, whose slope is below 1.1, by 1.1 of s's error and (1.5 |s| + 7) u of itself, and its slope, whose own slope
is below 0.51, by 0.51 of s's error and (3 |s| + 14) u (open + |s| open (1 - open)).  A gradient of an input is a sum of K + 1 such products, one of a weight of as many as there are steps, n:
the products' errors and n u of the sum of their magnitudes.  A result is rounded to its type once."""
import ctypes
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
ROUNDING = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
SMALLEST = {"f32": 2.0 ** -126, "bf16": 2.0 ** -126, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def rgc():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_1808_04357_amd as pkg
    pkg.load_library()
    return pkg


@pytest.fixture(scope="module")
def ctx(rgc):
    c = rgc.Context(1024, 1)
    yield c
    c.close()


def dtype_of(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[name]


def reference(x, weight, bias, silu, lengths, resets, before, dy, dlast):
    """Results and their bounds; every step looks back over its text by itself."""
    batch, steps, width = x.shape
    taps = weight.shape[1]
    keep = taps - 1
    n = np.full(batch, steps) if lengths is None else np.clip(lengths, 0, steps)
    out = {"y": np.zeros_like(x), "last": np.zeros((batch, keep, width)), "dx": np.zeros_like(x), "dweight": np.zeros_like(weight), "dbias": np.zeros(width),
           "dbefore": np.zeros((batch, keep, width))}
    slack = {k: np.zeros_like(v) for k, v in out.items()}
    size_w, size_b = np.zeros_like(weight), np.zeros(width)
    for b in range(batch):
        old = np.zeros((keep, width)) if before is None else before[b]
        line = np.concatenate([old, x[b, :n[b]]])                 # input t is at keep + t
        dline, eline, sizes = np.zeros_like(line), np.zeros_like(line), np.zeros_like(line)
        begin = -keep                                             # of the text
        for t in range(n[b]):
            if resets is not None and resets[b, t]:
                begin = t
            js = [j for j in range(taps) if t - keep + j >= begin]
            s = np.zeros(width) if bias is None else bias.copy()
            a = np.abs(s)
            for j in js:
                s = s + weight[:, j] * line[t + j]
                a = a + np.abs(weight[:, j] * line[t + j])
            e = 1.01 * taps * U * a
            o = 1 / (1 + np.exp(-s)) if silu else np.ones_like(s)
            h = 1 - o
            out["y"][b, t] = s * o
            slack["y"][b, t] = 1.1 * e + (1.5 * np.abs(s) + 7) * U * np.abs(s * o) if silu else e
            if dy is None:
                continue
            ds = dy[b, t] * (o * (1 + s * h) if silu else 1.0)
            eds = np.abs(dy[b, t]) * (0.51 * e + (3 * np.abs(s) + 14) * U * (o + np.abs(s) * o * h)) if silu else np.zeros_like(ds)
            for j in js:
                dline[t + j] += weight[:, j] * ds
                eline[t + j] += np.abs(weight[:, j]) * eds
                sizes[t + j] += np.abs(weight[:, j] * ds)
                out["dweight"][:, j] += ds * line[t + j]
                slack["dweight"][:, j] += eds * np.abs(line[t + j])
                size_w[:, j] += np.abs(ds * line[t + j])
            out["dbias"] += ds
            slack["dbias"] += eds
            size_b += np.abs(ds)
        last = [i for i in range(keep) if n[b] - keep + i >= begin]
        for i in last:
            out["last"][b, i] = line[n[b] + i]
        if dy is None:
            continue
        if dlast is not None:
            for i in last:
                dline[n[b] + i] += dlast[b, i]
                sizes[n[b] + i] += np.abs(dlast[b, i])
        eline += 1.01 * (taps + 1) * U * sizes
        out["dx"][b, :n[b]], slack["dx"][b, :n[b]] = dline[keep:], eline[keep:]
        out["dbefore"][b], slack["dbefore"][b] = dline[:keep], eline[:keep]
    slack["dweight"] += 1.01 * (int(n.sum()) + 1) * U * size_w
    slack["dbias"] += 1.01 * (int(n.sum()) + 1) * U * size_b
    return out, slack


def place(v, dtype, layout):
    import torch
    batch, steps, width = v.shape
    kind = dtype_of(dtype)
    if layout == "batch":
        t = torch.empty(batch, steps, width, dtype=kind, device="cuda")
    elif layout == "time":
        t = torch.empty(steps, batch, width, dtype=kind, device="cuda").transpose(0, 1)
    else:                                                # a part of a wider tensor, at an odd place
        t = torch.full((batch, steps, 2 * width + 5), 5.0, dtype=kind, device="cuda")[..., width + 1:2 * width + 1]
    t.copy_(torch.from_numpy(v))
    return t


def check(rgc, ctx, batch, steps, width, taps=4, dtype="f32", layout="batch", silu=True, bias=True, lengths=None, resets=None, state=True, train=True, seed=0, garbage=False,
          in_place=False, stream=None, dlast=True):
    import torch
    g = np.random.default_rng(seed + 1000 * steps + width)
    normal = lambda *s: g.standard_normal(s).astype(np.float32)      # noqa: E731
    x, dy, weight = normal(batch, steps, width), normal(batch, steps, width), normal(width, taps)
    if garbage:
        gone = np.arange(steps)[None] >= np.clip(lengths, 0, steps)[:, None]
        x[gone], dy[gone] = np.nan, np.inf
    put = lambda v, kind: None if v is None else torch.tensor(np.asarray(v), dtype=kind, device="cuda")   # noqa: E731
    kind = dtype_of(dtype)
    d_x, y = place(x, dtype, layout), place(np.full_like(x, 5.0), dtype, layout)
    d_w, d_b = put(weight, torch.float32), put(normal(width), torch.float32) if bias else None
    before = put(normal(batch, taps - 1, width), kind) if state else None
    old = before.clone() if state else None
    last = before if in_place else torch.full((batch, taps - 1, width), 5.0, dtype=kind, device="cuda") if state else None
    call = rgc.Convolution(d_x, d_w, y, bias=d_b, silu=silu, lengths=put(lengths, torch.int32), resets=put(resets, torch.uint8), before=before, last=last)
    torch.cuda.synchronize()
    rgc.rgc_causal_convolution(ctx, call, stream)
    got = {"y": y}
    if state:
        got["last"] = last
    d_dy = place(dy, dtype, layout) if train else None
    d_last = put(normal(batch, taps - 1, width), kind) if train and dlast else None
    if train:
        got.update(dx=place(np.full_like(x, 5.0), dtype, layout), dweight=torch.full((width, taps), 5.0, device="cuda"), dbefore=torch.full((batch, taps - 1, width), 5.0, dtype=kind, device="cuda"))
        if bias:
            got["dbias"] = torch.full((width,), 5.0, device="cuda")
        torch.cuda.synchronize()
        rgc.rgc_causal_convolution_backward(ctx, call, rgc.ConvolutionGrads(call, d_dy, got["dx"], got["dweight"], dbias=got.get("dbias"), dlast=d_last, dbefore=got["dbefore"]), stream)
    torch.cuda.synchronize()
    back = lambda t: None if t is None else t.double().cpu().numpy()    # noqa: E731
    want, slack = reference(back(d_x), back(d_w), back(d_b), silu, lengths, resets, back(old), back(d_dy), back(d_last))
    for k, t in got.items():
        a, w, r = back(t), want[k], "f32" if k in ("dweight", "dbias") else dtype
        ok = np.abs(a - w) <= 1.01 * ROUNDING[r] * np.abs(w) + slack[k] + np.where(slack[k] > 0, SMALLEST[r], 0.0)
        assert ok.all(), "%s: %d of %d off, first %r for %r (%r) at %r" % (k, (~ok).sum(), ok.size, a[~ok][0], w[~ok][0], slack[k][~ok][0], np.argwhere(~ok)[0])
    if layout == "slice":
        for k in ("y",) + (("dx",) if train else ()):
            whole = got[k]._base
            assert bool((whole[..., :width + 1] == 5.0).all()) and bool((whole[..., 2 * width + 1:] == 5.0).all())
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,steps,width", [(1, 1, 1), (64, 1, 1_500), (3, 1, 65), (2, 2, 3), (5, 7, 129), (20, 35, 300), (2, 15, 64), (1, 16, 2), (1, 17, 257), (2, 63, 7), (2, 64, 5),
                                               (1, 65, 70), (2, 67, 4), (1, 300, 33), (1, 1_000, 6)])
def test_every_length(rgc, ctx, dtype, batch, steps, width):
    check(rgc, ctx, batch, steps, width, dtype=dtype)


@pytest.mark.parametrize("taps", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("steps", [1, 5, 70])
def test_taps(rgc, ctx, taps, silu, steps):
    g = np.random.default_rng(steps)
    resets = (g.random((3, steps)) < 0.1).astype(np.uint8)
    check(rgc, ctx, 3, steps, 37, taps, "f32", silu=silu, bias=silu)
    check(rgc, ctx, 3, steps, 37, taps, "bf16", "slice", silu=silu, state=silu, resets=resets, lengths=np.array([steps, steps // 2, 0]), garbage=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["batch", "time", "slice"])
@pytest.mark.parametrize("width", [1, 3, 4, 66, 259])
def test_layouts(rgc, ctx, dtype, layout, width):
    check(rgc, ctx, 3, 70, width, 4, dtype, layout)


@pytest.mark.parametrize("steps", [1, 2, 20, 64, 129])
@pytest.mark.parametrize("taps", [2, 4, 8])
def test_rows_of_different_lengths(rgc, ctx, steps, taps):
    g = np.random.default_rng(steps)
    lengths = np.concatenate([[0, 1, 2, steps, steps + 7, -3, steps - 1, min(64, steps), min(65, steps), min(61, steps)], g.integers(0, steps + 1, 4)])
    for state in (True, False):
        check(rgc, ctx, len(lengths), steps, 9, taps, "f32", lengths=lengths, state=state, garbage=True)
    check(rgc, ctx, len(lengths), steps, 9, taps, "f16", "time", lengths=lengths, garbage=True, dlast=False)


@pytest.mark.parametrize("steps", [1, 3, 20, 64, 200])
@pytest.mark.parametrize("taps", [2, 4, 8])
def test_texts_packed_into_rows(rgc, ctx, steps, taps):
    g = np.random.default_rng(steps)
    resets = (g.random((7, steps)) < 0.2).astype(np.uint8)
    resets[0], resets[1], resets[3] = 0, 1, 0
    resets[2, 0] = 7
    resets[3, [t for t in (15, 16, 17, 61, 62, 63, 64, 65) if t < steps]] = 255
    resets[4, -1:] = 1
    resets[5, -2:] = [1, 0][-min(2, steps):]
    check(rgc, ctx, 7, steps, 10, taps, "f32", resets=resets)
    check(rgc, ctx, 7, steps, 10, taps, "bf16", resets=resets, lengths=np.array([steps, 3, 0, steps, steps // 2, steps - 1, 1]), garbage=True)


def test_inputs_before_a_text_do_not_matter_whatever_they_are(rgc, ctx):
    import torch
    x = torch.full((1, 40, 8), math.nan, device="cuda")
    x[:, 20:] = 1.0
    resets = torch.zeros(1, 40, dtype=torch.uint8, device="cuda")
    resets[0, 20] = 1
    y, last = torch.empty_like(x), torch.empty(1, 3, 8, device="cuda")
    before = torch.full((1, 3, 8), math.inf, device="cuda")
    call = rgc.Convolution(x, torch.ones(8, 4, device="cuda"), y, resets=resets, before=before, last=last)
    rgc.rgc_causal_convolution(ctx, call)
    assert y[0, 20:, 0].tolist() == [1.0, 2.0, 3.0] + [4.0] * 17 and bool((last == 1.0).all())
    dy, dx, dw, dbefore = torch.ones_like(x), torch.empty_like(x), torch.empty(8, 4, device="cuda"), torch.empty(1, 3, 8, device="cuda")
    rgc.rgc_causal_convolution_backward(ctx, call, rgc.ConvolutionGrads(call, dy, dx, dw, dbefore=dbefore))
    assert dx[0, :, 0].tolist() == [4.0] * 17 + [3.0, 2.0, 1.0] + [4.0] * 17 + [3.0, 2.0, 1.0] and dbefore[0, :, 0].tolist() == [1.0, 2.0, 3.0]


def test_no_rows_and_no_steps(rgc, ctx):
    check(rgc, ctx, 3, 0, 9, 4, "bf16")
    check(rgc, ctx, 3, 0, 9, 3, "f32", in_place=True)
    got = check(rgc, ctx, 0, 5, 9, 4, "f32")
    assert not got["dweight"].any() and not got["dbias"].any()


def test_one_token_at_a_time_in_place(rgc, ctx):
    """A prompt and the tokens after it, one by one with the kept inputs in place, give what the whole text gives."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    for dtype, taps, width in ((torch.bfloat16, 4, 301), (torch.float32, 2, 258), (torch.float16, 8, 3)):
        x, w = torch.randn(3, 30, width, generator=g, device="cuda").to(dtype), torch.randn(width, taps, generator=g, device="cuda")
        whole, parts = torch.empty_like(x), torch.empty_like(x)
        end, kept = torch.empty(3, taps - 1, width, dtype=dtype, device="cuda"), torch.zeros(3, taps - 1, width, dtype=dtype, device="cuda")
        rgc.rgc_causal_convolution(ctx, rgc.Convolution(x, w, whole, silu=True, last=end))
        rgc.rgc_causal_convolution(ctx, rgc.Convolution(x[:, :17], w, parts[:, :17], silu=True, last=kept))
        for t in range(17, 30):
            rgc.rgc_causal_convolution(ctx, rgc.Convolution(x[:, t:t + 1], w, parts[:, t:t + 1], silu=True, before=kept, last=kept))
        torch.cuda.synchronize()
        assert torch.equal(whole, parts) and torch.equal(end, kept)


def test_gradients_are_those_of_differences(rgc, ctx):
    """Central differences in the direction of the gradient itself: f(x + d g) - f(x - d g) = 2 d |g|^2 to d^2."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    batch, steps, width, taps = 2, 70, 5, 4
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    inputs = {"x": rand(batch, steps, width), "weight": rand(width, taps), "bias": rand(width), "before": rand(batch, taps - 1, width)}
    dy, dlast, y, last = rand(batch, steps, width), rand(batch, taps - 1, width), torch.empty(batch, steps, width, device="cuda"), torch.empty(batch, taps - 1, width, device="cuda")

    def call(t):
        return rgc.Convolution(t["x"], t["weight"], y, bias=t["bias"], silu=True, before=t["before"], last=last)

    def value(t):
        rgc.rgc_causal_convolution(ctx, call(t))
        return float((y.double() * dy.double()).sum() + (last.double() * dlast.double()).sum())

    c = call(inputs)
    rgc.rgc_causal_convolution(ctx, c)
    grads = {k: torch.empty_like(v) for k, v in inputs.items()}
    rgc.rgc_causal_convolution_backward(ctx, c, rgc.ConvolutionGrads(c, dy, grads["x"], grads["weight"], dbias=grads["bias"], dlast=dlast, dbefore=grads["before"]))
    for k, v in grads.items():
        unit = v / v.double().norm().float()
        step = 2.0 ** -7
        difference = (value({**inputs, k: inputs[k] + step * unit}) - value({**inputs, k: inputs[k] - step * unit})) / (2 * step)
        # values of y to 20 u each over 2 steps of 2^-7 (700 of them: 700 * 20 * 2^-24 * 2^6 = 0.05 at worst), and the third derivative
        assert abs(difference - float(v.double().norm())) < 0.05 + 2e-3 * float(v.double().norm()), k


def test_captured_and_on_another_stream(rgc, ctx):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    for batch, steps in ((5, 1), (2, 300)):
        x, w, b = torch.randn(batch, steps, 70, generator=g, device="cuda").bfloat16(), torch.randn(70, 4, generator=g, device="cuda"), torch.randn(70, generator=g, device="cuda")
        dy = torch.randn(batch, steps, 70, generator=g, device="cuda").bfloat16()
        new = lambda: {"y": torch.empty_like(x), "dx": torch.empty_like(x), "dw": torch.empty_like(w), "db": torch.empty_like(b)}      # noqa: E731

        def both(o, stream):
            call = rgc.Convolution(x, w, o["y"], bias=b, silu=True)
            grads = rgc.ConvolutionGrads(call, dy, o["dx"], o["dw"], dbias=o["db"])
            rgc.rgc_causal_convolution(ctx, call, stream)
            rgc.rgc_causal_convolution_backward(ctx, call, grads, stream)

        out, stream = new(), torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            both(out, stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both(out, stream)
        for _ in range(4):
            x.normal_(generator=g), dy.normal_(generator=g), w.normal_(generator=g)
            graph.replay()
            torch.cuda.synchronize()
            eager = new()
            both(eager, torch.cuda.current_stream())
            torch.cuda.synchronize()
            for k in out:
                assert torch.equal(out[k], eager[k]), k
        del graph


def test_refusals(rgc, ctx):
    import torch
    from paper_1808_04357_amd import binding
    lib = rgc.load_library()
    x, y, w = torch.zeros(2, 6, 8, device="cuda"), torch.zeros(2, 6, 8, device="cuda"), torch.zeros(8, 4, device="cuda")
    kept = torch.zeros(2, 3, 8, device="cuda")
    call = rgc.Convolution(x, w, y, before=kept)
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    grads = rgc.ConvolutionGrads(call, y, dx, dw)

    def refused(**changes):
        a = binding.rgc_convolution.from_buffer_copy(call.desc)
        for k, v in changes.items():
            setattr(a, k, v)
        return lib.rgc_causal_convolution(ctx.handle, ctypes.byref(a), None), lib.rgc_causal_convolution_backward(ctx.handle, ctypes.byref(a), grads._ref, None)

    assert refused() == (0, 0)
    seq = binding.rgc_sequence
    for changes in (dict(batch=-1), dict(steps=-1), dict(batch=2 ** 31), dict(width=0), dict(width=2 ** 21), dict(taps=0), dict(taps=9), dict(dtype=3), dict(silu=2), dict(weight=None),
                    dict(weight=w.data_ptr() + 2), dict(x=seq(None, 48, 8)), dict(x=seq(x.data_ptr(), -48, 8)), dict(x=seq(x.data_ptr() + 2, 48, 8)), dict(before=kept.data_ptr() + 2),
                    dict(x=seq(x.data_ptr(), 2 ** 50, 8))):
        assert refused(**changes) == (-1, -1), changes
    for changes in (dict(y=seq(None, 48, 8)), dict(y=seq(y.data_ptr(), 8, 8)), dict(y=seq(y.data_ptr(), 48, 4)), dict(y=call.desc.x), dict(last=kept.data_ptr())):
        assert refused(**changes)[0] == -1, changes
    for bad in (lambda: rgc.Convolution(x, w.half(), y), lambda: rgc.Convolution(x, w, y.half()), lambda: rgc.Convolution(x, w, y, before=kept[:, :2]), lambda: rgc.Convolution(x, w[:7], y),
                lambda: rgc.Convolution(x, w, y, lengths=torch.zeros(2, device="cuda")), lambda: rgc.Convolution(x.transpose(1, 2), w, y), lambda: rgc.ConvolutionGrads(call, y, dx, dw[:, :3]),
                lambda: rgc.ConvolutionGrads(call, y, dx, dw, dlast=kept.half()), lambda: rgc.rgc_causal_convolution_backward(ctx, call, rgc.ConvolutionGrads(call, y, y, dw)),
                lambda: rgc.rgc_causal_convolution_backward(ctx, call, rgc.ConvolutionGrads(call, y, dx, dw, dlast=kept, dbefore=kept))):
        with pytest.raises(rgc.RgcError):
            bad()
    torch.cuda.synchronize()
