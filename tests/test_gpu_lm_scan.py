"""The selective scan and its gradients against the definition in 64 bits, step by step.

Tolerances.  u = 2^-24.  A step's size is off by 16 u of itself and by what the rounding of its argument v makes of it, 2 u |v| times the softplus's slope.  A decay, whose exponent size * a has
two roundings and a size's error (the sum of a stretch's sizes, of 80 numbers, 80 u), is off by r = |a| E_size + (84 |size a| + 4) u relative.  So a state's error obeys
E_t = a_t E_{t-1} + r a_t |h_{t-1}| + |B| (|x| E_size + 4 u |size x|) + 3 u (|h_t| + a_t |h_{t-1}| + |size B x|), computed beside the reference, and a state's gradient's obeys the same run the other
way. What is made of them follows by the product rule: |C| E, |B| E and so on, with n u of the sum of the magnitudes for a sum of n, and (1.5 |z| + 8) u for silu(z), (3 |z| + 14) u times its parts for
its slope. Half of all that again is allowed for products of errors; a result is rounded to its type once."""
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


def reference(t, groups, softplus, lengths, resets, train):
    """t: arrays in 64 bits by name, None where there is none.  Results and the bounds of their errors."""
    x, rate = t["x"], t["a"]
    batch, steps, width = x.shape
    states, each = rate.shape[1], width // groups
    n = np.full(batch, steps) if lengths is None else np.clip(lengths, 0, steps)
    there = np.arange(steps)[None] < n[:, None]
    anew = np.zeros((batch, steps), bool) if resets is None else (resets != 0) & there
    on = there[..., None]
    only = lambda v: np.where(on, v, 0.0)                                             # noqa: E731
    x, v, z = only(x), only(t["delta"]) + (0.0 if t["delta_bias"] is None else t["delta_bias"]), None if t["gate"] is None else only(t["gate"])
    size = np.logaddexp(v, 0.0) if softplus else v
    grow = 1 / (1 + np.exp(-v)) if softplus else np.ones_like(v)
    size = only(size)
    e_size = only(16 * U * np.abs(size) + 2 * U * np.abs(v) * grow)
    o = 1 / (1 + np.exp(-z)) if z is not None else None
    shown = z * o if z is not None else np.ones_like(x)
    e_shown = np.abs(shown) * (1.5 * np.abs(z) + 8) * U if z is not None else np.zeros_like(x)
    through = np.zeros(width) if t["d"] is None else t["d"]
    wide = lambda p: np.repeat(only(p).reshape(batch, steps, groups, states), each, axis=2)      # noqa: E731
    b, c = wide(t["b"]), wide(t["c"])
    h = np.zeros((batch, width, states)) if t["h0"] is None else t["h0"].copy()
    e = np.zeros_like(h)
    prior, e_prior, after, e_after = (np.empty((steps,) + h.shape) for _ in range(4))
    for s in range(steps):
        keep = ~anew[:, s, None, None]
        prior[s], e_prior[s] = h * keep, e * keep
        sz, ez = size[:, s, :, None], e_size[:, s, :, None]
        a = np.exp(sz * rate)
        r = np.abs(rate) * ez + (84 * np.abs(sz * rate) + 4) * U
        fed, xs = sz * b[:, s] * x[:, s, :, None], x[:, s, :, None]
        new = a * prior[s] + fed
        e_new = a * e_prior[s] + r * a * np.abs(prior[s]) + np.abs(b[:, s]) * (np.abs(xs) * ez + 4 * U * np.abs(sz * xs)) + 3 * U * (np.abs(new) + np.abs(a * prior[s]) + np.abs(fed))
        live = there[:, s, None, None]
        h, e = np.where(live, new, h), np.where(live, e_new, e)
        after[s], e_after[s] = h, e
    ch = c.transpose(1, 0, 2, 3)
    inner = (ch * after).sum(3).transpose(1, 0, 2) + through * x
    e_inner = ((np.abs(ch) * e_after).sum(3) + (states + 3) * U * np.abs(ch * after).sum(3)).transpose(1, 0, 2) + (states + 3) * U * np.abs(through * x)
    out = {"y": only(inner * shown), "h_last": h}
    slack = {"y": only(e_inner * np.abs(shown) + np.abs(inner) * e_shown + 2 * U * np.abs(inner * shown)), "h_last": e}
    if not train:
        return out, slack
    dy = only(t["dy"])
    dinner = dy * shown
    e_dinner = np.abs(dy) * e_shown + U * np.abs(dinner)
    g = np.zeros_like(h) if t["dh_last"] is None else t["dh_last"].copy()
    e = np.zeros_like(g)
    came, e_came, slow, e_slow = (np.zeros_like(x) for _ in range(4))
    da, e_da, s_da = (np.zeros_like(rate) for _ in range(3))
    db, dc, e_db, e_dc, s_db, s_dc = (np.zeros((batch, steps, groups, states)) for _ in range(6))
    by_group = lambda p: p.reshape(batch, groups, each, states).sum(2)                # noqa: E731
    for s in range(steps - 1, -1, -1):
        live = there[:, s, None, None]
        sz, ez = size[:, s, :, None], e_size[:, s, :, None]
        a = np.exp(sz * rate)
        r = np.abs(rate) * ez + (84 * np.abs(sz * rate) + 4) * U
        di, edi = dinner[:, s, :, None], e_dinner[:, s, :, None]
        d = g + di * c[:, s]
        ed = e + np.abs(c[:, s]) * edi + 3 * U * (np.abs(d) + np.abs(di * c[:, s]))
        fed = sz * x[:, s, :, None]
        e_fed = np.abs(x[:, s, :, None]) * ez + U * np.abs(fed)
        zero = lambda p: np.where(live, p, 0.0)                                       # noqa: E731
        db[:, s], e_db[:, s], s_db[:, s] = by_group(zero(fed * d)), by_group(zero(np.abs(fed) * ed + e_fed * np.abs(d))), by_group(zero(np.abs(fed * d)))
        dc[:, s], e_dc[:, s], s_dc[:, s] = by_group(zero(di * after[s])), by_group(zero(np.abs(di) * e_after[s] + edi * np.abs(after[s]))), by_group(zero(np.abs(di * after[s])))
        came[:, s] = zero(d * b[:, s]).sum(2)
        e_came[:, s] = zero(np.abs(b[:, s]) * ed + (states + 1) * U * np.abs(d * b[:, s])).sum(2)
        back = a * d
        e_back = a * ed + r * a * np.abs(d) + U * np.abs(back)
        lost = back * prior[s]
        e_lost = e_back * np.abs(prior[s]) + np.abs(back) * e_prior[s] + U * np.abs(lost)
        slow[:, s] = zero(lost * rate).sum(2)
        e_slow[:, s] = zero(np.abs(rate) * e_lost + (states + 4) * U * np.abs(lost * rate)).sum(2)
        da += zero(lost * sz).sum(0)
        e_da += zero(e_lost * np.abs(sz) + np.abs(lost) * ez).sum(0)
        s_da += zero(np.abs(lost * sz)).sum(0)
        keep = ~anew[:, s, None, None]
        g, e = np.where(live, back * keep, g), np.where(live, e_back * keep, e)
    count = int(n.sum()) + 1
    dsize = came * x + slow
    e_dsize = np.abs(x) * e_came + e_slow + 4 * U * (np.abs(came * x) + np.abs(slow))
    dv = only(dsize * grow)
    e_dv = only(e_dsize * grow + np.abs(dsize * grow) * ((16 + 2 * np.abs(v)) * U if softplus else U))
    out.update(dx=only(came * size + dinner * through), ddelta=dv, da=da, db=db.reshape(batch, steps, groups * states), dc=dc.reshape(batch, steps, groups * states), dd=(dinner * x).sum((0, 1)),
               ddelta_bias=dv.sum((0, 1)), dh0=g)
    slack.update(dx=only(e_came * np.abs(size) + np.abs(came) * e_size + e_dinner * np.abs(through) + 3 * U * (np.abs(came * size) + np.abs(dinner * through))), ddelta=e_dv,
                 da=e_da + count * U * s_da, db=(e_db + (each + 1) * U * s_db).reshape(batch, steps, groups * states), dc=(e_dc + (each + 1) * U * s_dc).reshape(batch, steps, groups * states),
                 dd=(e_dinner * np.abs(x)).sum((0, 1)) + count * U * np.abs(dinner * x).sum((0, 1)), ddelta_bias=e_dv.sum((0, 1)) + count * U * np.abs(dv).sum((0, 1)), dh0=e)
    if z is not None:
        slope = o * (1 + z * (1 - o))
        out["dgate"] = only(dy * inner * slope)
        slack["dgate"] = only(np.abs(dy) * (e_inner * np.abs(slope) + np.abs(inner) * (3 * np.abs(z) + 14) * U * (o + np.abs(z) * o * (1 - o))) + 3 * U * np.abs(dy * inner * slope))
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


def check(rgc, ctx, batch, steps, width, states=16, groups=1, dtype="f32", layout="batch", gate=True, d=True, bias=True, softplus=True, lengths=None, resets=None, h0=True, train=True, seed=0,
          garbage=False, in_place=False, dh_last=True, stream=None, size=0.02):
    import torch
    g = np.random.default_rng(seed + 1000 * steps + width)
    normal = lambda *s: g.standard_normal(s).astype(np.float32)      # noqa: E731
    host = {"x": normal(batch, steps, width), "delta": 0.5 * normal(batch, steps, width), "b": normal(batch, steps, groups * states), "c": normal(batch, steps, groups * states),
            "gate": normal(batch, steps, width) if gate else None, "dy": normal(batch, steps, width)}
    if not softplus:
        host["delta"] = np.abs(host["delta"]) * 0.1
    if garbage:                                          # what lies behind a row's end is not looked at
        gone = np.arange(steps)[None] >= np.clip(lengths, 0, steps)[:, None]
        for k, v in host.items():
            if v is not None:
                v[gone] = np.nan if k != "c" else np.inf
    put = lambda v, kind: None if v is None else torch.tensor(np.asarray(v), dtype=kind, device="cuda")   # noqa: E731
    f32 = torch.float32
    t = {k: None if v is None else place(v, dtype, layout) for k, v in host.items()}
    t["a"] = put(-(np.arange(states) % 16 + 1) * (0.5 + g.random((width, states))), f32)
    t["d"] = put(normal(width), f32) if d else None
    t["delta_bias"] = put(np.log(np.expm1(size * np.exp(2.0 * g.random(width)))) if softplus else np.full(width, 0.01), f32) if bias else None
    t["h0"] = put(normal(batch, width, states), f32) if h0 else None
    t["dh_last"] = put(normal(batch, width, states), f32) if dh_last else None
    old = t["h0"].clone() if h0 else None
    five = lambda *s: torch.full(s, 5.0, device="cuda")              # noqa: E731
    like = lambda: place(np.full((batch, steps, width), 5.0, np.float32), dtype, layout)      # noqa: E731
    got = {"y": like(), "h_last": t["h0"] if in_place else five(batch, width, states)}
    kept = five(batch, -(-steps // rgc.RGC_SCAN_CHUNK), width, states) if train else None
    call = rgc.Scan(t["x"], t["delta"], t["a"], t["b"], t["c"], got["y"], groups=groups, d=t["d"], gate=t["gate"], delta_bias=t["delta_bias"], softplus=softplus,
                    lengths=put(lengths, torch.int32), resets=put(resets, torch.uint8), h0=t["h0"], h_last=got["h_last"], states=kept)
    torch.cuda.synchronize()
    rgc.rgc_selective_scan(ctx, call, stream)
    if train:
        row = lambda: place(np.full((batch, steps, groups * states), 5.0, np.float32), dtype, layout)      # noqa: E731
        got.update(dx=like(), ddelta=like(), db=row(), dc=row(), da=five(width, states), dd=five(width), ddelta_bias=five(width), dh0=five(batch, width, states))
        if gate:
            got["dgate"] = like()
        torch.cuda.synchronize()
        grads = rgc.ScanGrads(call, t["dy"], got["dx"], got["ddelta"], got["da"], got["db"], got["dc"], dd=got["dd"], dgate=got.get("dgate"), ddelta_bias=got["ddelta_bias"],
                              dh_last=t["dh_last"], dh0=got["dh0"])
        rgc.rgc_selective_scan_backward(ctx, call, grads, stream)
    torch.cuda.synchronize()
    back = lambda v: None if v is None else v.double().cpu().numpy()    # noqa: E731
    want, slack = reference({k: back(old if k == "h0" else v) for k, v in t.items()}, groups, softplus, lengths, resets, train)
    in_type = ("y", "dx", "ddelta", "dgate", "db", "dc")
    for k, v in got.items():
        a, w, kind = back(v), want[k], dtype if k in in_type else "f32"
        ok = np.abs(a - w) <= 1.01 * ROUNDING[kind] * np.abs(w) + 1.5 * slack[k] + np.where(slack[k] > 0, SMALLEST[kind], 0.0)
        assert ok.all(), "%s: %d of %d off, first %r for %r (%r) at %r" % (k, (~ok).sum(), ok.size, a[~ok][0], w[~ok][0], slack[k][~ok][0], np.argwhere(~ok)[0])
        if layout == "slice" and k in in_type:
            whole, n = v._base, v.shape[2]
            assert bool((whole[..., :n + 1] == 5.0).all()) and bool((whole[..., 2 * n + 1:] == 5.0).all()), k
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch,steps,width", [(1, 1, 1), (64, 1, 100), (3, 1, 65), (2, 2, 3), (5, 7, 129), (4, 8, 16), (3, 9, 17), (20, 35, 70), (2, 63, 33), (2, 64, 16), (2, 65, 15), (1, 72, 5),
                                               (3, 127, 4), (2, 128, 64), (1, 129, 40), (1, 1_000, 18), (1, 5_000, 2)])
def test_every_length(rgc, ctx, dtype, batch, steps, width):
    check(rgc, ctx, batch, steps, width, dtype=dtype)


@pytest.mark.parametrize("states", [1, 2, 3, 4, 5, 8, 9, 16, 17, 24, 25, 32, 33, 63, 64])
@pytest.mark.parametrize("groups", [1, 3])
@pytest.mark.parametrize("steps", [1, 20, 150])
def test_states_and_groups(rgc, ctx, states, groups, steps):
    check(rgc, ctx, 2, steps, 69, states, groups, "f32")
    check(rgc, ctx, 2, steps, 21, states, groups, "bf16", "slice", gate=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("layout", ["batch", "time", "slice"])
@pytest.mark.parametrize("states", [1, 7, 16, 24, 64])
def test_layouts(rgc, ctx, dtype, layout, states):
    check(rgc, ctx, 3, 70, 66, states, 2, dtype, layout)


@pytest.mark.parametrize("gate", [True, False])
@pytest.mark.parametrize("d", [True, False])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("softplus", [True, False])
def test_what_a_call_may_leave_out(rgc, ctx, gate, d, bias, softplus):
    for steps in (1, 10, 140):
        check(rgc, ctx, 2, steps, 20, 8, 1, "f32", gate=gate, d=d, bias=bias, softplus=softplus, h0=gate, dh_last=bias)


@pytest.mark.parametrize("steps,states", [(1, 16), (20, 4), (64, 16), (70, 1), (300, 16), (700, 64)])
def test_rows_of_different_lengths(rgc, ctx, steps, states):
    g = np.random.default_rng(steps)
    lengths = np.concatenate([[0, 1, steps, steps + 7, -3, steps - 1, min(64, steps), min(65, steps), min(8, steps)], g.integers(0, steps + 1, 4)])
    for h0 in (True, False):
        check(rgc, ctx, len(lengths), steps, 17, states, lengths=lengths, h0=h0, garbage=True)
    check(rgc, ctx, len(lengths), steps, 18, states, 2, "bf16", "time", lengths=lengths, garbage=True, dh_last=False)


@pytest.mark.parametrize("steps,states", [(1, 16), (20, 4), (64, 16), (70, 1), (300, 16), (700, 24)])
def test_states_that_start_anew(rgc, ctx, steps, states):
    g = np.random.default_rng(steps)
    resets = (g.random((6, steps)) < 0.05).astype(np.uint8)
    resets[0], resets[1], resets[3] = 0, 1, 0
    resets[2, 0] = 7
    resets[3, [t for t in (7, 8, 9, 63, 64, 65, 127, 128) if t < steps]] = 255
    for dtype in ("f32", "bf16"):
        check(rgc, ctx, 6, steps, 18, states, 1, dtype, resets=resets)
    check(rgc, ctx, 6, steps, 18, states, 2, "f32", "time", resets=resets, lengths=np.array([steps, 3, 0, steps, steps // 2, 1]), garbage=True)


def test_many_sequences_are_not_cut(rgc, ctx):
    """As many as fill the device: another walk than that of few long ones."""
    g = np.random.default_rng(1)
    check(rgc, ctx, 200, 70, 64, 16, 1, "f32", lengths=g.integers(0, 71, 200), resets=(g.random((200, 70)) < 0.02).astype(np.uint8), garbage=True)


def test_wide_and_slow(rgc, ctx):
    """Stretches of several chunks, and decays that reach over all of them."""
    check(rgc, ctx, 1, 700, 1_000, 16, 1, "bf16", train=False, size=0.0005)
    check(rgc, ctx, 2, 200, 700, 4, 1, "f32", size=0.0005)


def test_sizes_far_out(rgc, ctx):
    """Steps of no size, and of large ones: the softplus from -200 to 100."""
    import torch
    steps, width = 100, 6
    delta = torch.linspace(-200.0, 100.0, steps * width, device="cuda").view(1, steps, width)
    x, a = torch.ones(1, steps, width, device="cuda"), torch.full((width, 4), -1e-3, device="cuda")
    b = torch.ones(1, steps, 4, device="cuda")
    y, h = torch.empty_like(x), torch.empty(1, width, 4, device="cuda")
    kept = torch.empty(1, -(-steps // rgc.RGC_SCAN_CHUNK), width, 4, device="cuda")
    call = rgc.Scan(x, delta, a, b, b, y, softplus=True, h_last=h, states=kept)
    rgc.rgc_selective_scan(ctx, call)
    out = [torch.empty_like(x), torch.empty_like(x), torch.empty_like(a), torch.empty_like(b), torch.empty_like(b)]
    rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, torch.ones_like(x), *out))
    leaf = delta.double().cpu().requires_grad_()
    size, state, ys = torch.nn.functional.softplus(leaf, threshold=60.0), torch.zeros(width, dtype=torch.float64), []
    for t in range(steps):
        state = torch.exp(size[0, t] * float(a[0, 0])) * state + size[0, t]
        ys.append(4.0 * state)
    want = torch.stack(ys)[None]
    want.sum().backward()
    # 100 steps, each off by the 100 u that the head allows at most for |a| size < 0.1
    assert torch.allclose(y.double().cpu(), want.detach(), rtol=1e4 * U, atol=1e-30)
    assert torch.allclose(out[1].double().cpu(), leaf.grad, rtol=1e4 * U, atol=1e-30)


@pytest.mark.parametrize("steps", [33, 47, 48, 49])
@pytest.mark.parametrize("states", [8, 24, 32, 33])
def test_a_few_steps_more_than_a_chunk(rgc, ctx, steps, states):
    resets = np.random.default_rng(steps).random((4, steps)) < 0.1
    check(rgc, ctx, 4, steps, 21, states, 1, "f32", lengths=np.array([steps, 32, 33, steps - 1], np.int32), garbage=True, resets=resets)


def test_states_that_grow(rgc, ctx):
    """A factor over many steps may be beyond all numbers where no state is."""
    import torch
    steps, width, states = 600, 5, 16
    fives = lambda *s: torch.full(s, 5.0, device="cuda")             # noqa: E731
    x, dy = torch.zeros(1, steps, width, device="cuda"), torch.zeros(1, steps, width, device="cuda")
    delta, a, b = torch.ones_like(x), torch.full((width, states), 12.0, device="cuda"), torch.ones(1, steps, states, device="cuda")
    x[:, -3:], dy[:, :3] = 1.0, 1.0                                  # nothing but zeros is what grows
    y, h, kept = fives(1, steps, width), fives(1, width, states), fives(1, -(-steps // rgc.RGC_SCAN_CHUNK), width, states)
    call = rgc.Scan(x, delta, a, b, b, y, h_last=h, states=kept)
    rgc.rgc_selective_scan(ctx, call)
    dx, dv, da, db, dc, dh0 = fives(1, steps, width), fives(1, steps, width), fives(width, states), fives(1, steps, states), fives(1, steps, states), fives(1, width, states)
    rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, dy, dx, dv, da, db, dc, dh0=dh0))
    e = math.exp(12.0)
    after = [1.0, 1.0 + e, 1.0 + e + e * e]
    assert not y[0, :-3].any() and torch.allclose(y[0, -3:, 0].cpu().double(), torch.tensor(after, dtype=torch.float64) * states, rtol=1000 * U)
    assert torch.allclose(h.cpu().double(), torch.full((1, width, states), after[2], dtype=torch.float64), rtol=1000 * U)
    assert not dx[0, 3:].any() and torch.allclose(dx[0, :3, 0].cpu().double(), torch.tensor(after[::-1], dtype=torch.float64) * states, rtol=1000 * U)
    assert torch.allclose(dh0.cpu().double(), torch.full((1, width, states), e * after[2], dtype=torch.float64), rtol=1000 * U)
    assert not dv.any() and not da.any() and not db.any() and not dc.any()
    # what is small grows by exp(150) within a chunk; exponents of up to 150 are off by (80 + 4) u of themselves
    h0, dh_last = torch.full((1, width, states), 1e-37, device="cuda"), torch.full((1, width, states), 2e-37, device="cuda")
    x.zero_(), dy.zero_(), delta.zero_(), a.fill_(1.0)
    delta[:, 32:64] = 150.0 / 32.0
    call = rgc.Scan(x, delta, a, b, b, y, h0=h0, h_last=h, states=kept)
    rgc.rgc_selective_scan(ctx, call)
    rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, dy, dx, dv, da, db, dc, dh_last=dh_last, dh0=dh0))
    for got, of in ((h, h0), (dh0, dh_last)):
        assert torch.allclose(got.cpu().double(), of.cpu().double() * math.exp(150.0), rtol=150 * 84 * 2 * U)


def test_infinite_rates_and_states(rgc, ctx):
    import torch
    x = torch.ones(1, 20, 2, device="cuda")
    delta, b = torch.full_like(x, 0.5), torch.ones(1, 20, 2, device="cuda")
    a = torch.tensor([[-math.inf, -1.0], [-1.0, -math.inf]], device="cuda")
    y, h = torch.empty_like(x), torch.full((1, 2, 2), 3.0, device="cuda")
    # steps behind the row's end leave the states as they are, whatever their rates
    rgc.rgc_selective_scan(ctx, rgc.Scan(x, delta, a, b, b, y, lengths=torch.tensor([0], dtype=torch.int32, device="cuda"), h0=h, h_last=h))
    assert bool((h == 3.0).all()) and not y.any()
    rgc.rgc_selective_scan(ctx, rgc.Scan(x, delta, a, b, b, y, lengths=torch.tensor([3], dtype=torch.int32, device="cuda"), h0=h, h_last=h))
    assert h[0, 0, 0] == 0.5 and h[0, 1, 1] == 0.5 and h[0, 0, 1] > 1.0 and not y[0, 3:].any()
    # an infinite state is no part of what begins after it
    h[0, 0, 0] = math.inf
    resets = torch.zeros(1, 20, dtype=torch.uint8, device="cuda")
    resets[0, 9] = 1
    rgc.rgc_selective_scan(ctx, rgc.Scan(x, delta, -torch.ones(2, 2, device="cuda"), b, b, y, resets=resets, h0=h, h_last=h))
    assert bool(torch.isinf(y[0, :9, 0]).all()) and bool(torch.isfinite(y[0, 9:]).all()) and bool(torch.isfinite(y[0, :, 1]).all()) and bool(torch.isfinite(h).all())


def test_no_rows_and_no_steps(rgc, ctx):
    import torch
    check(rgc, ctx, 3, 0, 9, 5, dtype="bf16")
    got = check(rgc, ctx, 0, 5, 9, 5)
    assert not got["da"].any() and not got["dd"].any()


def test_one_token_at_a_time_in_place(rgc, ctx):
    """A prompt and the tokens after it, one by one with the state in place, give what the whole text gives, to the states' errors (cut differently, they round differently)."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(1)
    for states, width in ((16, 33), (1, 70), (64, 5)):
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
        x, delta, z, b, c = rand(3, 90, width), rand(3, 90, width), rand(3, 90, width), rand(3, 90, states), rand(3, 90, states)
        a = -torch.rand(width, states, generator=g, device="cuda")
        whole, parts, end, state = torch.empty_like(x), torch.empty_like(x), torch.empty(3, width, states, device="cuda"), torch.zeros(3, width, states, device="cuda")
        rgc.rgc_selective_scan(ctx, rgc.Scan(x, delta, a, b, c, whole, gate=z, softplus=True, h_last=end))

        def go(first, upto):
            cut = lambda t: t[:, first:upto]      # noqa: E731
            rgc.rgc_selective_scan(ctx, rgc.Scan(cut(x), cut(delta), a, cut(b), cut(c), cut(parts), gate=cut(z), softplus=True, h0=state, h_last=state))

        go(0, 70)
        for t in range(70, 90):
            go(t, t + 1)
        torch.cuda.synchronize()
        assert torch.allclose(whole, parts, rtol=1e-5, atol=1e-4) and torch.allclose(end, state, rtol=1e-5, atol=1e-5)


def test_same_bits_every_time(rgc, ctx):
    import torch
    for steps, width in ((300, 100), (30, 200)):
        first = check(rgc, ctx, 2, steps, width, dtype="bf16", seed=4)
        for _ in range(2):
            again = check(rgc, ctx, 2, steps, width, dtype="bf16", seed=4)
            for k in first:
                assert torch.equal(first[k], again[k]), k


def test_gradients_are_those_of_differences(rgc, ctx):
    """Central differences in the direction of each gradient: f(v + s g) - f(v - s g) = 2 s |g|^2 to s^2."""
    import torch
    g = torch.Generator(device="cuda").manual_seed(2)
    batch, steps, width, states = 2, 70, 6, 4
    rand = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
    inputs = {"x": rand(batch, steps, width), "delta": rand(batch, steps, width) - 2.0, "a": -torch.rand(width, states, generator=g, device="cuda") - 0.1, "b": rand(batch, steps, states),
              "c": rand(batch, steps, states), "d": rand(width), "gate": rand(batch, steps, width), "delta_bias": rand(width), "h0": rand(batch, width, states)}
    dy, dh, y, h = rand(batch, steps, width), rand(batch, width, states), torch.empty(batch, steps, width, device="cuda"), torch.empty(batch, width, states, device="cuda")
    kept = torch.empty(batch, -(-steps // rgc.RGC_SCAN_CHUNK), width, states, device="cuda")

    def call(t):
        return rgc.Scan(t["x"], t["delta"], t["a"], t["b"], t["c"], y, d=t["d"], gate=t["gate"], delta_bias=t["delta_bias"], softplus=True, h0=t["h0"], h_last=h, states=kept)

    def value(t):
        rgc.rgc_selective_scan(ctx, call(t))
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    c = call(inputs)
    rgc.rgc_selective_scan(ctx, c)
    grads = {k: torch.empty_like(v) for k, v in inputs.items()}
    rgc.rgc_selective_scan_backward(ctx, c, rgc.ScanGrads(c, dy, grads["x"], grads["delta"], grads["a"], grads["b"], grads["c"], dd=grads["d"], dgate=grads["gate"],
                                                          ddelta_bias=grads["delta_bias"], dh_last=dh, dh0=grads["h0"]))
    for k, v in grads.items():
        norm = float(v.double().norm())
        unit, step = v / norm, 2.0 ** -8
        difference = (value({**inputs, k: inputs[k] + step * unit}) - value({**inputs, k: inputs[k] - step * unit})) / (2 * step)
        # 840 outputs of a few units, each to some 50 u, over two steps of 2^-8: 840 * 4 * 50 * 2^-24 * 2^7 = 1.3 were all errors to add up, 0.05 as they do not
        assert abs(difference - norm) < 0.05 + 4e-3 * norm, (k, difference, norm)


def test_captured_and_on_another_stream(rgc, ctx):
    import torch
    g = torch.Generator(device="cuda").manual_seed(3)
    for batch, steps, width in ((5, 1, 40), (2, 30, 40), (1, 600, 70)):
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")      # noqa: E731
        seqs = {k: rand(batch, steps, width) for k in ("x", "delta", "gate", "dy")}
        seqs.update({k: rand(batch, steps, 16) for k in ("b", "c")})
        a = -torch.rand(width, 16, generator=g, device="cuda")
        kept = torch.empty(batch, -(-steps // rgc.RGC_SCAN_CHUNK), width, 16, device="cuda")
        new = lambda: {k: torch.empty_like(v) for k, v in (("y", seqs["x"]), ("dx", seqs["x"]), ("ddelta", seqs["x"]), ("dgate", seqs["x"]), ("da", a), ("db", seqs["b"]), ("dc", seqs["b"]))}      # noqa: E731

        def both(o, stream):
            call = rgc.Scan(seqs["x"], seqs["delta"], a, seqs["b"], seqs["c"], o["y"], gate=seqs["gate"], softplus=True, states=kept)
            rgc.rgc_selective_scan(ctx, call, stream)
            rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, seqs["dy"], o["dx"], o["ddelta"], o["da"], o["db"], o["dc"], dgate=o["dgate"]), stream)

        out, stream = new(), torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            both(out, stream)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            both(out, stream)
        for _ in range(4):
            for v in seqs.values():
                v.normal_(generator=g)
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
    zeros = lambda *s: torch.zeros(*s, device="cuda")      # noqa: E731
    x, delta, b, c, y, a = zeros(2, 6, 8), zeros(2, 6, 8), zeros(2, 6, 4), zeros(2, 6, 4), zeros(2, 6, 8), zeros(8, 4)
    call = rgc.Scan(x, delta, a, b, c, y, states=zeros(2, 1, 8, 4))
    grads = rgc.ScanGrads(call, x, zeros(2, 6, 8), zeros(2, 6, 8), zeros(8, 4), zeros(2, 6, 4), zeros(2, 6, 4))

    def refused(**changes):
        s = binding.rgc_scan.from_buffer_copy(call.desc)
        for k, v in changes.items():
            setattr(s, k, v)
        return lib.rgc_selective_scan(ctx.handle, ctypes.byref(s), None), lib.rgc_selective_scan_backward(ctx.handle, ctypes.byref(s), grads._ref, None)

    assert refused() == (0, 0)
    seq = binding.rgc_sequence
    for changes in (dict(batch=-1), dict(steps=-1), dict(batch=2 ** 31), dict(width=0), dict(width=2 ** 21), dict(states=0), dict(states=65), dict(groups=0), dict(groups=3), dict(groups=9), dict(dtype=3),
                    dict(softplus=2), dict(a=None), dict(a=a.data_ptr() + 2), dict(x=seq(None, 48, 8)), dict(delta=seq(None, 48, 8)), dict(b=seq(None, 24, 4)), dict(c=seq(None, 24, 4)),
                    dict(b=seq(b.data_ptr(), -24, 4)), dict(x=seq(x.data_ptr() + 2, 48, 8)), dict(gate=seq(x.data_ptr() + 1, 48, 8)), dict(h0=a.data_ptr() + 1), dict(x=seq(x.data_ptr(), 2 ** 50, 8))):
        assert refused(**changes) == (-1, -1), changes
    far = 2 ** 27 + 1                                                 # of steps: a tile's are addressed by 32 bits
    for changes in (dict(x=seq(x.data_ptr(), 8, far)), dict(delta=seq(x.data_ptr(), 8, far)), dict(b=seq(b.data_ptr(), 4, far)), dict(c=seq(c.data_ptr(), 4, far))):
        assert refused(**changes) == (-1, -1), changes
    for changes in (dict(y=seq(None, 48, 8)), dict(y=seq(y.data_ptr(), 8, 8)), dict(y=seq(y.data_ptr(), 48, 4)), dict(y=seq(y.data_ptr(), 8, far)), dict(y=call.desc.x), dict(y=call.desc.delta),
                    dict(gate=call.desc.y)):
        assert refused(**changes)[0] == -1, changes
    for changes in (dict(kept=None), dict(gate=call.desc.x)):          # (no place for the gate's gradient)
        assert refused(**changes)[1] == -1, changes
    b2, c2 = zeros(2, 6, 4), zeros(2, 6, 4)
    backward = lambda dy, dx, dv, db, dc: rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, dy, dx, dv, zeros(8, 4), db, dc))      # noqa: E731
    for bad in (lambda: rgc.Scan(x, delta, a, b[..., :3], c, y), lambda: rgc.Scan(x, delta.half(), a, b, c, y), lambda: rgc.Scan(x, delta, a.half(), b, c, y), lambda: rgc.Scan(x, delta, a, b, c, y, groups=3),
                lambda: rgc.Scan(x, delta, a, b, c, y, groups=2), lambda: rgc.Scan(x, delta, a, b, c, y, h0=zeros(2, 8)), lambda: rgc.Scan(x, delta, a, b, c, y, states=zeros(2, 2, 8, 4)),
                lambda: rgc.Scan(x, delta, a, b, c, y, resets=zeros(2, 6)), lambda: rgc.ScanGrads(call, x, y, y, a, b, c, dgate=y), lambda: rgc.ScanGrads(call, x, y, y, a[:7], b, c), lambda: backward(x, y, y, b2, c2), lambda: backward(x, x, y, b2, c2),
                lambda: backward(x, y, zeros(2, 6, 8), b2, b2), lambda: backward(x, y, zeros(2, 6, 8), b, c2)):
        with pytest.raises(rgc.RgcError):
            bad()
    torch.cuda.synchronize()
