"""What is measured of a selective state space language model's own operators: the calls that a program makes which trains or serves one
around the gradient compression, from the tokens to the layers' states, one case each.

A case names its operator (``kind``) and the call's sizes and options.  Kinds:

  embed  rgc_embed_tokens (with ``train``: then rgc_embed_tokens_backward, the table's dense gradient as the compressor takes it)
  conv   rgc_causal_convolution (with ``train``: then rgc_causal_convolution_backward)
  scan   rgc_selective_scan (with ``train``: then rgc_selective_scan_backward)

``left_out``: the share of positions that are padding (tokens of -1).  ``state``: the call takes what an earlier one kept, and keeps it.
Inputs lie as a program has them: as parts of one product's output, which makes rows strided.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}


def _embed(name, rows, vocab, width, **options):
    case = {"name": name, "kind": "embed", "rows": rows, "vocab": vocab, "width": width, "dtype": "bf16", "table_dtype": "bf16", "scale": 1.0,
            "left_out": 0.0, "train": False}
    case.update(options)
    return case


def _conv(name, batch, steps, width, **options):
    case = {"name": name, "kind": "conv", "batch": batch, "steps": steps, "width": width, "taps": 4, "dtype": "bf16", "time_major": False,
            "silu": True, "lengths": False, "resets": False, "state": False, "train": False}
    case.update(options)
    return case


def _scan_case(name, batch, steps, width, **options):
    case = {"name": name, "kind": "scan", "batch": batch, "steps": steps, "width": width, "states": 16, "groups": 1, "dtype": "bf16",
            "time_major": False, "gate": True, "lengths": False, "resets": False, "state": False, "train": False}
    case.update(options)
    return case


def listed():
    return [
        # the next token of 64 streams: the recurrent model's vocabulary and width
        _embed("embed_one_token", 64, 10_000, 1_500, dtype="f32", table_dtype="f32"),
        # a training step of the recurrent model: 20 streams of 35 tokens
        _embed("embed_lstm_step", 700, 10_000, 1_500, dtype="f32", table_dtype="f32", train=True),
        # reading long prompts with a scaled table of odd width
        _embed("embed_prompts", 32_768, 33_278, 1_501, dtype="f16", table_dtype="f16", scale=math.sqrt(1_501.0)),
        # a training step of a large batch, one position in ten is padding; the weights in 32 bits, the activations in 16
        _embed("embed_training", 32_768, 50_257, 2_048, table_dtype="f32", left_out=0.1, train=True),
        # one decoding step of 64 streams
        _conv("conv_one_token", 64, 1, 1_500, state=True),
        # reading one long prompt, the last inputs are kept for the tokens after it
        _conv("conv_prompt", 1, 32_768, 1_500, state=True),
        # training on long rows into which several texts are packed
        _conv("conv_packed_training", 8, 4_096, 2_048, resets=True, train=True),
        # one decoding step of 64 streams: one token each, state in, state out
        _scan_case("scan_one_token", 64, 1, 1_500, state=True),
        # truncated back-propagation: 20 streams of 35 steps, time first
        _scan_case("scan_lstm_step", 20, 35, 1_500, dtype="f32", time_major=True, state=True, train=True),
        # reading one long prompt
        _scan_case("scan_prompt", 1, 32_768, 1_500, state=True),
        # a batch of texts of different lengths, an odd width, B and C of two groups of channels with more states each
        _scan_case("scan_ragged_training", 6, 1_001, 1_502, dtype="f16", states=24, groups=2, lengths=True, train=True),
        # training on long rows into which several texts are packed
        _scan_case("scan_packed_training", 8, 4_096, 2_048, resets=True, train=True),
    ]


# the most that a drawn case has: bytes of any kind, and states of a scan over all its steps
_MOST_BYTES, _MOST_STATES = 1_000_000_000, 1_050_000_000


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["embed", "conv", "scan", "scan"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    train = rng.random() < 0.5
    if kind == "embed":
        case = _embed("", _log_uniform(rng, 1, 65_536), _log_uniform(rng, 1_000, 200_000), _log_uniform(rng, 64, 4_096), dtype=dtype,
                      table_dtype=rng.choice([dtype, "f32"]), scale=rng.choice([1.0, 0.5, 12.25]), left_out=rng.choice([0.0, 0.0, 0.3]), train=train)
        size = "rows"
    else:
        batch, width = _log_uniform(rng, 1, 128), _log_uniform(rng, 64, 4_096)
        steps = 1 if rng.random() < 0.15 else _log_uniform(rng, 2, 32_768)
        common = dict(dtype=dtype, time_major=rng.random() < 0.3, lengths=rng.random() < 0.3, resets=rng.random() < 0.3, state=rng.random() < 0.5, train=train)
        if kind == "conv":
            case = _conv("", batch, steps, width, taps=rng.choice([2, 3, 4, 4]), silu=rng.random() < 0.8, **common)
        else:
            groups = rng.choice([1, 1, 1, 2, 4])
            case = _scan_case("", batch, steps, -(-width // groups) * groups, groups=groups, states=rng.choice([1, 4, 8, 16, 16, 24, 32, 64]),
                              gate=rng.random() < 0.7, **common)
        size = "steps"
    del case["name"]
    while work(case)["bytes"] > _MOST_BYTES and case[size] > 1:
        case[size] = max(1, int(case[size] * min(0.95, _MOST_BYTES / work(case)["bytes"])))
    if work(case)["bytes"] > _MOST_BYTES:                        # a table, or many streams' states
        smaller = "vocab" if kind == "embed" else "batch"
        case[smaller] = max(1, int(case[smaller] * 0.95 * _MOST_BYTES / work(case)["bytes"]))
    if kind == "scan":
        many = case["batch"] * case["steps"] * case["width"] * case["states"] / _MOST_STATES
        if many > 1.0:
            case["steps"] = max(1, int(case["steps"] / many))
    return case


def _different(tokens, vocab):
    """How many words so many tokens are, as _embed_inputs draws them: the n-th with probability ln((n + 1) / n) / ln(vocab + 1).  (In stretches of
    words about as frequent as each other.)"""
    first, found = 1, 0.0
    while first <= vocab:
        end = min(vocab + 1, first + max(1, first // 16))
        p = math.log(end / first) / math.log(vocab + 1.0) / (end - first)
        found += (end - first) * -math.expm1(tokens * math.log1p(-p))
        first = end
    return found


def work(case):
    s, train = _SIZE[case["dtype"]], case["train"]
    if case["kind"] == "embed":
        # a row of the table is read once however many tokens want it
        n, tokens = case["rows"] * case["width"], case["rows"] * (1.0 - case["left_out"])
        table = _different(tokens, case["vocab"]) * case["width"]
        moved = 4 * case["rows"] + table * _SIZE[case["table_dtype"]] + n * s
        if train:
            moved += tokens * case["width"] * s + case["vocab"] * case["width"] * 4
        return {"bytes": float(moved), "flops": float(n * (2 if train else 1))}
    batch, steps, width = case["batch"], case["steps"], case["width"]
    n = batch * steps * width
    masks = (batch * steps if case["resets"] else 0) + (4 * batch if case["lengths"] else 0)
    if case["kind"] == "conv":
        taps = case["taps"]
        moved = n * s * (4 if train else 2) + 4 * width * (taps + 1) * (2 if train else 1) + masks
        moved += batch * (taps - 1) * width * s * ((4 if train else 2) if case["state"] else 0)
        return {"bytes": float(moved), "flops": float(n * (2 * taps + 5) * (3 if train else 1))}
    states, groups, gate = case["states"], case["groups"], 1 if case["gate"] else 0
    tensors = 3 + gate + ((3 + gate) if train else 0)
    moved = n * s * tensors + 2 * batch * steps * groups * states * s * (2 if train else 1) + masks
    moved += 4 * width * (states + 2) * (2 if train else 1) + 4 * batch * width * states * ((4 if train else 2) if case["state"] else 0)
    # a state's step: the decay, its power, what comes in, what goes out; backward the states again, their gradients, and five products with those
    return {"bytes": float(moved), "flops": float(n * states * (7 + (20 if train else 0)) + n * (15 + (30 if train else 0)))}


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _embed_inputs(case, seed):
    """Tokens as texts have them: the n-th frequent word about once in n."""
    g, dev = _generator(seed), "cuda"
    rows, vocab, width = case["rows"], case["vocab"], case["width"]
    rank = (torch.rand(rows, generator=g, device=dev, dtype=torch.float64) * math.log(vocab + 1.0)).exp().long() - 1
    tokens = torch.randperm(vocab, generator=g, device=dev)[rank.clamp(0, vocab - 1)]
    if case["left_out"]:
        tokens = torch.where(torch.rand(rows, generator=g, device=dev) < case["left_out"], torch.full_like(tokens, -1), tokens)
    state = {"case": case, "tokens": tokens.to(torch.int32),
             "table": (torch.randn(vocab, width, generator=g, device=dev) * 0.05).to(_DTYPES[case["table_dtype"]])}
    if case["train"]:
        state["dout"] = (torch.randn(rows, width, generator=g, device=dev) * 0.01).to(_DTYPES[case["dtype"]])
    return state


def _sequences(case, g):
    """Makers of [batch, steps, n] tensors as the case lays them out, and what says which steps there are."""
    dev, dtype, batch, steps = "cuda", _DTYPES[case["dtype"]], case["batch"], case["steps"]

    def normal(n, spread=1.0):
        lead = (steps, batch) if case["time_major"] else (batch, steps)
        t = (torch.randn(*lead, n, generator=g, device=dev) * spread).to(dtype)
        return t.transpose(0, 1) if case["time_major"] else t

    masks = {"lengths": None, "resets": None}
    if case["lengths"]:
        masks["lengths"] = torch.randint(0, steps + 1, (batch,), generator=g, device=dev).to(torch.int32)
    if case["resets"]:
        masks["resets"] = (torch.rand(batch, steps, generator=g, device=dev) < 1.0 / 300.0).to(torch.uint8)
    return normal, masks


def _conv_inputs(case, seed):
    g, dev = _generator(seed), "cuda"
    batch, width, taps = case["batch"], case["width"], case["taps"]
    normal, state = _sequences(case, g)
    state.update(case=case, projected=normal(2 * width),          # the layer's inputs and its gates: one product's output
                 weight=torch.randn(width, taps, generator=g, device=dev) * taps ** -0.5, bias=torch.randn(width, generator=g, device=dev) * 0.1)
    kept = lambda: torch.randn(batch, taps - 1, width, generator=g, device=dev).to(_DTYPES[case["dtype"]])      # noqa: E731
    state["before"] = kept() if case["state"] else None
    if case["train"]:
        state["dy"], state["dlast"] = normal(width), kept() if case["state"] else None
    return state


def _scan_inputs(case, seed):
    """Decays of one to some hundred steps, as such layers begin: rates of 1 to `states`, step sizes of 0.001 to 0.1."""
    g, dev = _generator(seed), "cuda"
    batch, width, states, groups = case["batch"], case["width"], case["states"], case["groups"]
    normal, state = _sequences(case, g)
    rank = -(-width // 16)
    size = (torch.rand(width, generator=g, device=dev) * math.log(100.0)).exp() * 0.001
    state.update(case=case, x=normal(width), delta=normal(width, 0.5), mixed=normal(rank + 2 * groups * states),     # one product's output: delta's factor, B and C
                 projected=normal(2 * width) if case["gate"] else None,
                 a=-torch.arange(1, states + 1, device=dev).float() * (0.5 + torch.rand(width, states, generator=g, device=dev)),
                 d=torch.randn(width, generator=g, device=dev), delta_bias=size + torch.log(-torch.expm1(-size)))
    kept = lambda: torch.randn(batch, width, states, generator=g, device=dev)      # noqa: E731
    state["h0"] = kept() if case["state"] else None
    if case["train"]:
        state["dy"], state["dh_last"] = normal(width), kept() if case["state"] else None
    return state


def _b_and_c(state):
    rank, n = -(-state["case"]["width"] // 16), state["case"]["groups"] * state["case"]["states"]
    return state["mixed"][..., rank:rank + n], state["mixed"][..., rank + n:]


_INPUTS = {"embed": _embed_inputs, "conv": _conv_inputs, "scan": _scan_inputs}
_handle = []


def _context(rgc):
    """The program's one context (made at the first call)."""
    if not _handle:
        _handle.append(rgc.Context(1 << 16, 1))
    return _handle[0]


def prepare(case, seed):
    state = _INPUTS[case["kind"]](case, seed)
    if not own:
        return state
    # what a program keeps: the context, the output buffers, and the call's descriptor over both
    import paper_1808_04357_amd as rgc
    dev, dtype, out = "cuda", _DTYPES[case["dtype"]], {}
    state["rgc"], state["ctx"], state["stream"], state["out"] = rgc, _context(rgc), torch.cuda.current_stream(), out

    def f32(*shape):
        return torch.empty(*shape, dtype=torch.float32, device=dev)

    if case["kind"] == "embed":
        out["out"] = torch.empty(case["rows"], case["width"], dtype=dtype, device=dev)
        state["call"] = rgc.Embedding(state["table"], state["tokens"], out["out"], scale=case["scale"])
        if case["train"]:
            out["dtable"] = f32(case["vocab"], case["width"])
        return state
    batch, steps, width = case["batch"], case["steps"], case["width"]

    def sequence(n):
        lead = (steps, batch) if case["time_major"] else (batch, steps)
        t = torch.empty(*lead, n, dtype=dtype, device=dev)
        return t.transpose(0, 1) if case["time_major"] else t

    out["y"] = sequence(width)
    if case["kind"] == "conv":
        taps = case["taps"]

        def kept():
            return torch.empty(batch, taps - 1, width, dtype=dtype, device=dev) if case["state"] else None

        out["last"] = kept()
        state["call"] = rgc.Convolution(state["projected"][..., :width], state["weight"], out["y"], bias=state["bias"], silu=case["silu"],
                                        lengths=state["lengths"], resets=state["resets"], before=state["before"], last=out["last"])
        if case["train"]:
            out.update(dx=sequence(width), dweight=f32(width, taps), dbias=f32(width), dbefore=kept())
            state["grads"] = rgc.ConvolutionGrads(state["call"], state["dy"], out["dx"], out["dweight"], dbias=out["dbias"], dlast=state["dlast"],
                                                  dbefore=out["dbefore"])
        return state
    states, groups = case["states"], case["groups"]
    b, c = _b_and_c(state)
    gate = state["projected"][..., width:] if case["gate"] else None
    out["h_last"] = f32(batch, width, states) if case["state"] else None
    kept = f32(batch, -(-steps // rgc.RGC_SCAN_CHUNK), width, states) if case["train"] else None
    state["call"] = rgc.Scan(state["x"], state["delta"], state["a"], b, c, out["y"], groups=groups, d=state["d"], gate=gate, delta_bias=state["delta_bias"],
                             softplus=True, lengths=state["lengths"], resets=state["resets"], h0=state["h0"], h_last=out["h_last"], states=kept)
    if case["train"]:
        out.update(dx=sequence(width), ddelta=sequence(width), da=f32(width, states), db=sequence(groups * states), dc=sequence(groups * states),
                   dd=f32(width), dgate=sequence(width) if case["gate"] else None, ddelta_bias=f32(width),
                   dh0=f32(batch, width, states) if case["state"] else None)
        state["grads"] = rgc.ScanGrads(state["call"], state["dy"], out["dx"], out["ddelta"], out["da"], out["db"], out["dc"], dd=out["dd"],
                                       dgate=out["dgate"], ddelta_bias=out["ddelta_bias"], dh_last=state["dh_last"], dh0=out["dh0"])
    return state


# ------------------------------------------------------------------------------------------------ the calls

def run(state):
    if own:
        return _call(state)
    return {"embed": _plain_embed, "conv": _plain_conv, "scan": _plain_scan}[state["case"]["kind"]](state)


def _call(state):
    rgc, case, ctx, stream, out = state["rgc"], state["case"], state["ctx"], state["stream"], state["out"]
    if case["kind"] == "embed":
        rgc.rgc_embed_tokens(ctx, state["call"], stream)
        if case["train"]:
            rgc.rgc_embed_tokens_backward(ctx, state["call"], state["dout"], out["dtable"], rgc.RGC_OVERWRITE, stream)
    elif case["kind"] == "conv":
        rgc.rgc_causal_convolution(ctx, state["call"], stream)
        if case["train"]:
            rgc.rgc_causal_convolution_backward(ctx, state["call"], state["grads"], stream)
    else:
        rgc.rgc_selective_scan(ctx, state["call"], stream)
        if case["train"]:
            rgc.rgc_selective_scan_backward(ctx, state["call"], state["grads"], stream)
    return {k: v for k, v in out.items() if v is not None}


# ------------------------------------------------------------------------------------------------ the plain forms

def _plain_embed(state):
    case, table, tokens = state["case"], state["table"], state["tokens"].long()
    there = ((tokens >= 0) & (tokens < case["vocab"]))[:, None]
    at = tokens.clamp(0, case["vocab"] - 1)
    rows = table[at].float() * case["scale"]
    out = {"out": torch.where(there, rows, torch.zeros_like(rows)).to(_DTYPES[case["dtype"]])}
    if case["train"]:
        dout = state["dout"].float()
        dout = torch.where(there, dout, torch.zeros_like(dout))
        out["dtable"] = torch.zeros(case["vocab"], case["width"], device=dout.device).index_add_(0, at, dout) * case["scale"]
    return out


def _there(state, like):
    """[batch, steps, 1]: whether the row has the step."""
    batch, steps = like.shape[:2]
    if state["lengths"] is None:
        return torch.ones(batch, steps, 1, dtype=torch.bool, device=like.device)
    return (torch.arange(steps, device=like.device) < state["lengths"][:, None])[..., None]


def _texts(state, kept, like):
    """[batch, kept + steps]: which of its row's texts each step belongs to, those before the first step too."""
    batch, steps = like.shape[:2]
    text = torch.zeros(batch, kept + steps, dtype=torch.int32, device=like.device)
    if state["resets"] is not None:
        text[:, kept:] = torch.cumsum(state["resets"] != 0, dim=1)
    return text


def _plain_conv(state):
    case, width, taps = state["case"], state["case"]["width"], state["case"]["taps"]
    steps, kept, dtype = case["steps"], taps - 1, _DTYPES[case["dtype"]]
    x, weight = state["projected"][..., :width].float(), state["weight"]
    there, text = _there(state, x), _texts(state, kept, x)
    x = torch.where(there, x, torch.zeros_like(x))
    before = torch.zeros_like(x[:, :1]).expand(-1, kept, -1) if state["before"] is None else state["before"].float()
    u = torch.cat([before, x], dim=1)
    same = [(text[:, j:j + steps] == text[:, kept:])[..., None] for j in range(taps)]
    s = state["bias"] + sum(weight[:, j] * torch.where(same[j], u[:, j:j + steps], torch.zeros_like(x)) for j in range(taps))
    opened = torch.sigmoid(s) if case["silu"] else torch.ones_like(s)
    y = torch.where(there, s * opened, torch.zeros_like(s))
    out = {"y": y.to(dtype)}
    n = torch.full_like(text[:, 0], steps).long() if state["lengths"] is None else state["lengths"].clamp(0, steps).long()
    if case["state"]:
        # the `kept` inputs that end with the row's last step, those of its last text
        at = n[:, None] + torch.arange(kept, device=n.device)
        final = text.gather(1, (n + kept - 1)[:, None])
        lasts = (text.gather(1, at) == final)[..., None]
        at = at[..., None].expand(-1, -1, width)
        out["last"] = torch.where(lasts, u.gather(1, at), torch.zeros_like(u[:, :kept])).to(dtype)
    if case["train"]:
        slope = opened * (1.0 + s * (1.0 - opened)) if case["silu"] else torch.ones_like(s)
        ds = torch.where(there, state["dy"].float() * slope, torch.zeros_like(s))
        du = torch.zeros_like(u)
        if case["state"]:
            du.scatter_add_(1, at, torch.where(lasts, state["dlast"].float(), torch.zeros_like(u[:, :kept])))
        dweight = torch.empty_like(weight)
        for j in range(taps):
            part = torch.where(same[j], ds, torch.zeros_like(ds))
            du[:, j:j + steps] += weight[:, j] * part
            dweight[:, j] = (part * u[:, j:j + steps]).sum(dim=(0, 1))
        out["dx"] = torch.where(there, du[:, kept:], torch.zeros_like(ds)).to(dtype)
        out.update(dweight=dweight, dbias=ds.sum(dim=(0, 1)))
        if case["state"]:
            out["dbefore"] = du[:, :kept].to(dtype)
    return out


def _joined(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, from h = 0: every pass joins stretches twice as long.  (Overwrites both.)"""
    step = 1
    while step < b.shape[1]:
        b[:, step:] += a[:, step:] * b[:, :-step]
        a[:, step:] = a[:, step:] * a[:, :-step]
        step *= 2
    return b


def _plain_scan(state):
    case, width, steps, groups, states = state["case"], state["case"]["width"], state["case"]["steps"], state["case"]["groups"], state["case"]["states"]
    dtype, batch = _DTYPES[case["dtype"]], case["batch"]
    there = _there(state, state["x"])
    zero = lambda t: torch.where(there, t, torch.zeros_like(t))                      # noqa: E731
    x, v = zero(state["x"].float()), zero(state["delta"].float()) + state["delta_bias"]
    b, c = (zero(t.float()).reshape(batch, steps, groups, 1, states) for t in _b_and_c(state))
    size = zero(torch.where(v > 20.0, v, torch.log1p(torch.exp(v))))                 # (a step that is not there leaves the state as it is)
    if case["gate"]:
        z = zero(state["projected"][..., width:].float())
        opened = torch.sigmoid(z)
        shown = z * opened
    else:
        shown = torch.ones_like(x)

    def by_group(t):
        return t.reshape(batch, steps, groups, width // groups, -1)

    a = torch.exp(size[..., None] * state["a"])
    if state["resets"] is not None:
        a = a * ((state["resets"] == 0)[..., None] | ~there)[..., None]
    h = (by_group(size * x) * b).reshape(batch, steps, width, states)
    h0 = state["h0"] if case["state"] else torch.zeros_like(h[:, 0])
    h[:, 0] += a[:, 0] * h0
    h = _joined(a.clone(), h)
    inner = (by_group(h) * c).sum(dim=4).reshape(batch, steps, width) + state["d"] * x
    out = {"y": zero(inner * shown).to(dtype)}
    if case["state"]:
        out["h_last"] = h[:, -1].clone()
    if case["train"]:
        dy = zero(state["dy"].float())
        dinner = dy * shown
        d = (by_group(dinner) * c).reshape(batch, steps, width, states)
        out["dc"] = (by_group(dinner) * by_group(h)).sum(dim=3).reshape(batch, steps, -1).to(dtype)
        if case["state"]:
            d[:, -1] += state["dh_last"]
        after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], dim=1)
        d = _joined(after.flip(1), d.flip(1)).flip(1)
        out["db"] = zero((by_group(size * x) * by_group(d)).sum(dim=3).reshape(batch, steps, -1)).to(dtype)
        came = (by_group(d) * b).sum(dim=4).reshape(batch, steps, width)             # gradient of what comes in, size * x
        decay = d * a * torch.cat([h0[:, None], h[:, :-1]], dim=1)                   # gradient of the decay's exponent
        dsize = came * x + (decay * state["a"]).sum(dim=3)
        dv = zero(dsize * torch.sigmoid(v))
        out["dx"] = zero(came * size + dinner * state["d"]).to(dtype)
        out.update(ddelta=dv.to(dtype), da=(decay * size[..., None]).sum(dim=(0, 1)), dd=(dinner * x).sum(dim=(0, 1)), ddelta_bias=dv.sum(dim=(0, 1)))
        if case["gate"]:
            out["dgate"] = zero(dy * inner * opened * (1.0 + z * (1.0 - opened))).to(dtype)
        if case["state"]:
            out["dh0"] = a[:, 0] * d[:, 0]
    return out


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    with torch.no_grad():
        return {"embed": _exact_embed, "conv": _exact_conv, "scan": _exact_scan}[case["kind"]](case, _INPUTS[case["kind"]](case, seed))


def _exact_embed(case, t):
    token = t["tokens"].long()
    known = (token >= 0) & (token < case["vocab"])
    scale = float(torch.tensor(case["scale"], dtype=torch.float32))
    out = torch.zeros(case["rows"], case["width"], dtype=torch.float64, device="cuda")
    out[known] = t["table"][token[known]].double() * scale
    if not case["train"]:
        return {"out": out}
    dtable = torch.zeros(case["vocab"], case["width"], dtype=torch.float64, device="cuda")
    dtable.index_put_((token[known],), t["dout"][known].double() * scale, accumulate=True)
    return {"out": out, "dtable": dtable}


def _ends(case, t):
    """[batch] lengths, and [batch, steps] 1.0 where a row has the step."""
    n = torch.full((case["batch"],), case["steps"], device="cuda") if t["lengths"] is None else t["lengths"].long().clamp(0, case["steps"])
    return n, (torch.arange(case["steps"], device="cuda")[None] < n[:, None]).double()


def _exact_conv(case, t):
    """Tap by tap: how far back it reaches, and whether a text began since."""
    width, taps, steps, batch = case["width"], case["taps"], case["steps"], case["batch"]
    n, on = _ends(case, t)
    x, w = t["projected"][..., :width].double(), t["weight"].double()
    anew = torch.zeros(batch, steps, device="cuda", dtype=torch.bool) if t["resets"] is None else t["resets"] != 0
    # how many steps back the text of a step began (far back where it began before the row)
    began = torch.where(anew, torch.arange(steps, device="cuda")[None].expand(batch, -1), torch.full((batch, steps), -taps, device="cuda")).cummax(dim=1).values
    since = torch.arange(steps, device="cuda")[None] - began
    old = torch.zeros(batch, taps - 1, width, dtype=torch.float64, device="cuda") if t["before"] is None else t["before"].double()
    line = torch.cat([old, x], dim=1)

    def back(lag):
        return line[:, taps - 1 - lag:taps - 1 - lag + steps]

    def reach(lag):
        return ((since >= lag).double() * on)[..., None]

    s = t["bias"].double().expand(batch, steps, width).clone()
    for lag in range(taps):
        s += w[:, taps - 1 - lag] * back(lag) * reach(lag)
    gate = 1.0 / (1.0 + (-s).exp()) if case["silu"] else torch.ones_like(s)
    out = {"y": s * gate * on[..., None]}
    if case["state"]:
        at = n[:, None] + torch.arange(taps - 1, device="cuda")                       # on the line
        end = torch.where(n > 0, began.gather(1, (n - 1).clamp(min=0)[:, None])[:, 0], torch.full_like(n, -taps))
        mine = (at - (taps - 1) >= end[:, None]).double()[..., None]
        index = at[..., None].expand(-1, -1, width)
        out["last"] = line.gather(1, index) * mine
    if case["train"]:
        ds = t["dy"].double() * on[..., None] * (gate * (1.0 + s * (1.0 - gate)) if case["silu"] else 1.0)
        dline, dw = torch.zeros_like(line), torch.zeros_like(w)
        for lag in range(taps):
            dline[:, taps - 1 - lag:taps - 1 - lag + steps] += w[:, taps - 1 - lag] * ds * reach(lag)
            dw[:, taps - 1 - lag] = (ds * back(lag) * reach(lag)).sum(dim=(0, 1))
        if case["state"]:
            dline.scatter_add_(1, index, t["dlast"].double() * mine)
            out["dbefore"] = dline[:, :taps - 1]
        out.update(dx=dline[:, taps - 1:] * on[..., None], dweight=dw, dbias=ds.sum(dim=(0, 1)))
    return out


def _exact_scan(case, t):
    """Step by step, as the formula stands."""
    width, steps, batch, groups, states = case["width"], case["steps"], case["batch"], case["groups"], case["states"]
    _, on = _ends(case, t)
    rate, through = t["a"].double(), t["d"].double()
    each = width // groups
    x = t["x"].double() * on[..., None]
    v = t["delta"].double() + t["delta_bias"].double()
    size = torch.logaddexp(v, torch.zeros_like(v)) * on[..., None]
    mixed = t["mixed"].double()
    first = mixed.shape[-1] - 2 * groups * states
    b, c = (p.reshape(batch, steps, groups, states) for p in mixed[..., first:].split(groups * states, dim=2))
    carry = torch.ones_like(on) if t["resets"] is None else 1.0 - (t["resets"] != 0).double() * on
    z = t["projected"][..., width:].double() if case["gate"] else None
    gate = 1.0 / (1.0 + (-z).exp()) if case["gate"] else None

    def spread(p, s):                                                                 # [batch, groups, states] of a step to [batch, width, states]
        return p[:, s].repeat_interleave(each, dim=1)

    h = torch.zeros(batch, width, states, dtype=torch.float64, device="cuda") if t["h0"] is None else t["h0"].double()
    before = torch.empty(steps, batch, width, states, dtype=torch.float64, device="cuda") if case["train"] else None
    inner = torch.empty(batch, steps, width, dtype=torch.float64, device="cuda")
    fed = size * x
    for s in range(steps):
        h = h * carry[:, s, None, None]
        if case["train"]:
            before[s] = h
        h = (size[:, s, :, None] * rate).exp() * h + fed[:, s, :, None] * spread(b, s)
        inner[:, s] = (h * spread(c, s)).sum(dim=2)
    inner += through * x
    out = {"y": inner * (z * gate if case["gate"] else 1.0) * on[..., None]}
    if case["state"]:
        out["h_last"] = h
    if not case["train"]:
        return out
    dy = t["dy"].double() * on[..., None]
    if case["gate"]:
        out["dgate"] = dy * inner * gate * (1.0 + z * (1.0 - gate))
        dy = dy * z * gate
    d = torch.zeros_like(h) if t["dh_last"] is None else t["dh_last"].double().clone()
    came, dsize, da = torch.empty_like(inner), torch.empty_like(inner), torch.zeros_like(rate)
    db, dc = torch.empty_like(b), torch.empty_like(c)
    for s in range(steps - 1, -1, -1):
        there = on[:, s, None, None]
        decay = (size[:, s, :, None] * rate).exp()
        decayed = decay * before[s]
        now = decayed + fed[:, s, :, None] * spread(b, s)
        dc[:, s] = (dy[:, s, :, None] * now).reshape(batch, groups, each, states).sum(dim=2)
        d += dy[:, s, :, None] * spread(c, s) * there
        db[:, s] = (fed[:, s, :, None] * d).reshape(batch, groups, each, states).sum(dim=2)
        came[:, s] = (d * spread(b, s)).sum(dim=2)
        decayed *= d * there
        da += (decayed * size[:, s, :, None]).sum(dim=0)
        dsize[:, s] = (decayed * rate).sum(dim=2)
        d = d * decay * carry[:, s, None, None]
    dv = (came * x + dsize) * on[..., None] / (1.0 + (-v).exp())
    out.update(dx=(came * size + dy * through) * on[..., None], ddelta=dv, da=da, db=(db * on[..., None, None]).flatten(2), dc=dc.flatten(2),
               dd=(dy * x).sum(dim=(0, 1)), ddelta_bias=dv.sum(dim=(0, 1)))
    if case["state"]:
        out["dh0"] = d
    return out
