"""The embedding, the short convolution, the selective scan and the scores of tokens as a state space model runs them, training and serving; calls with tensors of far strides and of more rows than a
grid holds."""
import math

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rgc():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    import paper_1808_04357_amd as pkg
    pkg.load_library()
    return pkg


VOCAB, WIDTH, STATES, RANK, TAPS = 211, 24, 5, 3, 4
INNER = 2 * WIDTH


def parameters(seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s: torch.randn(*s, generator=g)      # noqa: E731
    return {"table": rand(VOCAB, WIDTH) * 0.3, "into": rand(WIDTH, 2 * INNER) * WIDTH ** -0.5, "taps": rand(INNER, TAPS) * 0.5, "tap_bias": rand(INNER) * 0.1,
            "mix": rand(INNER, RANK + 2 * STATES) * INNER ** -0.5, "size": rand(RANK, INNER) * RANK ** -0.5, "size_bias": rand(INNER) - 3.0,
            "rate": -torch.arange(1.0, STATES + 1).repeat(INNER, 1) * (0.5 + torch.rand(INNER, STATES, generator=g)), "through": rand(INNER), "out": rand(INNER, VOCAB) * INNER ** -0.5}


class Layers:
    """One layer's buffers and descriptors over [batch, steps] tokens."""

    def __init__(self, rgc, p, batch, steps, resets=None, kept=None, state=None):
        import torch
        self.rgc, self.p, self.n = rgc, p, batch * steps
        new = lambda *s: torch.empty(*s, device="cuda")      # noqa: E731
        self.tokens, self.targets = (torch.zeros(batch * steps, dtype=torch.int32, device="cuda") for _ in range(2))
        self.embedded, self.split, self.u, self.mixed = new(batch, steps, WIDTH), new(batch, steps, 2 * INNER), new(batch, steps, INNER), new(batch, steps, RANK + 2 * STATES)
        self.delta, self.y, self.logits = new(batch, steps, INNER), new(batch, steps, INNER), new(batch * steps, VOCAB)
        self.lookup = rgc.Embedding(p["table"], self.tokens, self.embedded.view(-1, WIDTH), scale=math.sqrt(WIDTH))
        x, z = self.split.split(INNER, dim=2)
        self.convolution = rgc.Convolution(x, p["taps"], self.u, bias=p["tap_bias"], silu=True, resets=resets, before=kept, last=kept)
        factor, b, c = self.mixed.split([RANK, STATES, STATES], dim=2)
        states = new(batch, -(-steps // rgc.RGC_SCAN_CHUNK), INNER, STATES)
        self.scan = rgc.Scan(self.u, self.delta, p["rate"], b, c, self.y, d=p["through"], gate=z, delta_bias=p["size_bias"], softplus=True, resets=resets, h0=state, h_last=state, states=states)
        self.logprob, self.stats = new(batch * steps), new(batch * steps, 2)
        self.scores = rgc.TokenScores(self.logits, self.targets, logprob=self.logprob, stats=self.stats)

    def forward(self, ctx, stream=None):
        import torch
        rgc, p = self.rgc, self.p
        rgc.rgc_embed_tokens(ctx, self.lookup, stream)
        torch.matmul(self.embedded, p["into"], out=self.split)
        rgc.rgc_causal_convolution(ctx, self.convolution, stream)
        torch.matmul(self.u, p["mix"], out=self.mixed)
        torch.matmul(self.mixed[..., :RANK], p["size"], out=self.delta)
        rgc.rgc_selective_scan(ctx, self.scan, stream)
        torch.matmul(self.y.view(-1, INNER), p["out"], out=self.logits)
        rgc.rgc_token_logprobs(ctx, self.scores, stream)

    def backward(self, ctx, weight, stream=None):
        """Gradients of sum(weight * logprob)."""
        import torch
        rgc, p = self.rgc, self.p
        g = {k: torch.empty_like(v) for k, v in p.items()}
        dlogits = torch.empty_like(self.logits)
        rgc.rgc_token_logprobs_backward(ctx, self.scores, dlogits, grad_logprob=weight, stream=stream)
        dy = (dlogits @ p["out"].t()).view_as(self.y)
        g["out"] = self.y.view(-1, INNER).t() @ dlogits
        dsplit, du, ddelta, dmixed = torch.empty_like(self.split), torch.empty_like(self.u), torch.empty_like(self.delta), torch.empty_like(self.mixed)
        dx, dz = dsplit.split(INNER, dim=2)
        dfactor, db, dc = dmixed.split([RANK, STATES, STATES], dim=2)
        rgc.rgc_selective_scan_backward(ctx, self.scan, rgc.ScanGrads(self.scan, dy, du, ddelta, g["rate"], db, dc, dd=g["through"], dgate=dz, ddelta_bias=g["size_bias"]), stream)
        dfactor.copy_(ddelta @ p["size"].t())
        g["size"] = self.mixed[..., :RANK].reshape(-1, RANK).t() @ ddelta.view(-1, INNER)
        g["mix"] = self.u.view(-1, INNER).t() @ dmixed.view(-1, RANK + 2 * STATES)
        du += dmixed @ p["mix"].t()
        rgc.rgc_causal_convolution_backward(ctx, self.convolution, rgc.ConvolutionGrads(self.convolution, du, dx, g["taps"], dbias=g["tap_bias"]), stream)
        g["into"] = self.embedded.view(-1, WIDTH).t() @ dsplit.view(-1, 2 * INNER)
        dembedded = (dsplit @ p["into"].t()).view(-1, WIDTH)
        rgc.rgc_embed_tokens_backward(ctx, self.lookup, dembedded, g["table"], rgc.RGC_OVERWRITE, stream)
        return g


def model64(p, tokens, resets):
    """Logits in 64 bits on the CPU, step by step; differentiable."""
    import torch
    batch, steps = tokens.shape
    known = (tokens >= 0)[..., None]
    e = torch.where(known, p["table"][tokens.clamp(min=0)] * math.sqrt(WIDTH), torch.zeros((), dtype=torch.float64))
    x, z = (e @ p["into"]).split(INNER, dim=2)
    rows = []
    for b in range(batch):
        h, begin, ys = torch.zeros(INNER, STATES, dtype=torch.float64), 0, []
        for t in range(steps):
            if resets is not None and resets[b, t]:
                h, begin = torch.zeros_like(h), t
            s = p["tap_bias"] + sum(p["taps"][:, j] * x[b, t - TAPS + 1 + j] for j in range(TAPS) if t - TAPS + 1 + j >= begin)
            u = torch.nn.functional.silu(s)
            factor, bb, cc = (u @ p["mix"]).split([RANK, STATES, STATES])
            size = torch.nn.functional.softplus(factor @ p["size"] + p["size_bias"])
            h = torch.exp(size[:, None] * p["rate"]) * h + (size * u)[:, None] * bb
            ys.append((h @ cc + p["through"] * u) * torch.nn.functional.silu(z[b, t]))
        rows.append(torch.stack(ys))
    return torch.stack(rows) @ p["out"]


@pytest.mark.parametrize("steps", [1, 13, 35, 70])
@pytest.mark.parametrize("packed", [False, True])
def test_training_step(rgc, steps, packed):
    import torch
    batch = 3
    host = parameters(1)
    p = {k: v.cuda() for k, v in host.items()}
    g = torch.Generator().manual_seed(steps)
    tokens, targets = torch.randint(0, VOCAB, (batch, steps), generator=g), torch.randint(0, VOCAB, (batch, steps), generator=g)
    tokens[0, 0] = targets[1, steps // 2] = -1
    resets = (torch.rand(batch, steps, generator=g) < 0.1) if packed else None
    weight = torch.randn(batch * steps, generator=g)
    ctx = rgc.Context(1, 1)
    layers = Layers(rgc, p, batch, steps, None if resets is None else resets.cuda())
    layers.tokens.copy_(tokens.view(-1)), layers.targets.copy_(targets.view(-1))
    layers.forward(ctx)
    got = layers.backward(ctx, weight.cuda())
    torch.cuda.synchronize()
    own = {k: v.double().requires_grad_() for k, v in host.items()}
    logits = model64(own, tokens, resets).view(-1, VOCAB)
    logprob = torch.log_softmax(logits, dim=1).gather(1, targets.view(-1, 1).clamp(min=0))[:, 0] * (targets.view(-1) >= 0)
    (logprob * weight).sum().backward()
    # fp32 products of 24 to 211 terms between the operators: some 1e-6 of the values
    assert torch.allclose(layers.logprob.cpu().double(), logprob.detach(), rtol=1e-4, atol=1e-4)
    for k, v in own.items():
        assert float((got[k].cpu().double() - v.grad).norm()) <= 1e-4 * float(v.grad.norm()) + 1e-9, k
    ctx.close()


def test_serving_token_by_token(rgc):
    """A prompt, then single tokens with the kept inputs and the states in place, in a graph that is replayed for each; against the whole text at once."""
    import torch
    batch, steps, prompt = 2, 60, 41
    p = {k: v.cuda() for k, v in parameters(2).items()}
    tokens = torch.randint(0, VOCAB, (batch, steps), generator=torch.Generator().manual_seed(9)).to(torch.int32).cuda()
    ctx, stream = rgc.Context(1, 1), torch.cuda.Stream()
    kept = torch.zeros(batch, TAPS - 1, INNER, device="cuda")
    state = torch.zeros(batch, INNER, STATES, device="cuda")
    whole = Layers(rgc, p, batch, steps)
    whole.tokens.copy_(tokens.reshape(-1))
    whole.forward(ctx)
    # (the prompt's `last` is a buffer of its own: in place is for single steps)
    first, one = Layers(rgc, p, batch, prompt, state=state), Layers(rgc, p, batch, 1, kept=kept, state=state)
    x = first.split[..., :INNER]
    first.convolution = rgc.Convolution(x, p["taps"], first.u, bias=p["tap_bias"], silu=True, last=kept)
    first.tokens.copy_(tokens[:, :prompt].reshape(-1))
    first.forward(ctx)
    said = first.logits.view(batch, prompt, VOCAB)[:, -1]
    torch.cuda.synchronize()
    assert torch.allclose(said, whole.logits.view(batch, steps, VOCAB)[:, prompt - 1], rtol=1e-4, atol=1e-4)
    stream.wait_stream(torch.cuda.current_stream())
    before = kept.clone(), state.clone()
    with torch.cuda.stream(stream):
        one.forward(ctx, stream)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        one.forward(ctx, stream)
    kept.copy_(before[0]), state.copy_(before[1])
    for t in range(prompt, steps):
        one.tokens.copy_(tokens[:, t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.allclose(one.logits, whole.logits.view(batch, steps, VOCAB)[:, t], rtol=1e-4, atol=2e-4), t
    del graph
    ctx.close()


def test_two_contexts_on_two_streams(rgc):
    """Calls of different contexts at once give what they give one after the other."""
    import torch
    p = {k: v.cuda() for k, v in parameters(3).items()}
    batch, steps = 4, 100
    weight = torch.randn(batch * steps, device="cuda")
    runs = []
    for seed in (1, 2):
        layers = Layers(rgc, p, batch, steps)
        layers.tokens.copy_(torch.randint(0, VOCAB, (batch * steps,), generator=torch.Generator().manual_seed(seed)))
        runs.append((layers, rgc.Context(1, 1), torch.cuda.Stream()))
    torch.cuda.synchronize()
    together = []
    for layers, ctx, stream in runs:
        with torch.cuda.stream(stream):
            layers.forward(ctx, stream)
            together.append(layers.backward(ctx, weight, stream))
    torch.cuda.synchronize()
    for (layers, ctx, _), got in zip(runs, together):
        layers.forward(ctx)
        alone = layers.backward(ctx, weight)
        torch.cuda.synchronize()
        for k in ("rate", "through", "size_bias", "taps", "tap_bias", "table"):      # (what the operators themselves write)
            assert torch.equal(alone[k], got[k]), k
        ctx.close()


def test_rows_that_lie_far_apart(rgc):
    """Strides that pass 2^31 elements."""
    import torch
    ctx, far = rgc.Context(1, 1), 2 ** 31 + 64
    memory = torch.zeros(far + 20_000, dtype=torch.bfloat16, device="cuda")
    near = torch.randn(2, 40, 30, device="cuda").bfloat16()
    wide = memory.as_strided((2, 40, 30), (far, 300, 1))
    wide.copy_(near)
    w, y = torch.randn(30, 4, device="cuda"), [torch.empty_like(near) for _ in range(2)]
    for x, to in zip((near, wide), y):
        rgc.rgc_causal_convolution(ctx, rgc.Convolution(x, w, to, silu=True))
    assert torch.equal(y[0], y[1])
    a, b = -torch.rand(30, 16, device="cuda"), torch.randn(2, 40, 16, device="cuda").bfloat16()
    grads = []
    for x, to in zip((near, wide), y):
        kept = torch.empty(2, 2, 30, 16, device="cuda")
        call = rgc.Scan(x, x, a, b, b, to, gate=x, softplus=True, states=kept)
        rgc.rgc_selective_scan(ctx, call)
        out = [torch.empty_like(near) for _ in range(3)] + [torch.empty_like(b) for _ in range(2)] + [torch.empty_like(a)]
        rgc.rgc_selective_scan_backward(ctx, call, rgc.ScanGrads(call, x, out[0], out[1], out[5], out[3], out[4], dgate=out[2]))
        grads.append(out)
    torch.cuda.synchronize()
    assert torch.equal(y[0], y[1]) and all(torch.equal(g, h) for g, h in zip(*grads))
    ctx.close()


def test_more_rows_than_a_grid_holds(rgc):
    """More workgroups than one launch takes."""
    import torch
    ctx, rows = rgc.Context(1, 1), 2 ** 24 + 4_099
    table = torch.randn(100, 4, device="cuda").half()
    tokens = (torch.arange(rows, device="cuda") % 101).to(torch.int32)                 # (100 is left out)
    out = torch.empty(rows, 4, dtype=torch.float16, device="cuda")
    rgc.rgc_embed_tokens(ctx, rgc.Embedding(table, tokens, out))
    torch.cuda.synchronize()
    want = torch.cat([table, torch.zeros(1, 4, device="cuda").half()])[tokens.long()]
    assert torch.equal(out, want)
    ctx.close()
