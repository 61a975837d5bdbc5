"""What is measured of the language-model operators: the calls a program makes that trains, distills or scores a
recurrent language model around the gradient compression, one case each.

A case names its operator (``kind``) and the call's sizes and options.  Kinds:

  score    rgc_token_logprobs (with ``train``: then rgc_token_logprobs_backward, as a policy step calls it)
  distill  rgc_distill_loss (with ``train``: loss and gradient in the one call)
  recur    rgc_gated_recurrence (with ``train``: then rgc_gated_recurrence_backward)

Rows are token positions.  ``pad`` columns behind the vocabulary hold NaN: they belong to the row's storage, not to the
row.  ``left_out``: the share of rows whose target is no token.  ``banned``: the share of a row's logits that are -inf.
"""
from __future__ import annotations

import math
import random

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f32": 4, "bf16": 2, "f16": 2}
_STATE_STEPS = 256         # the recurrence keeps its state once in so many steps for the backward pass (rgc.RGC_RECURRENCE_CHUNK)


def _score(name, rows, vocab, **options):
    case = {"name": name, "kind": "score", "rows": rows, "vocab": vocab, "pad": 0, "dtype": "bf16", "temperature": 1.0, "top": 0,
            "left_out": 0.0, "banned": 0.0, "train": False}
    case.update(options)
    return case


def _distill(name, rows, vocab, **options):
    case = {"name": name, "kind": "distill", "rows": rows, "vocab": vocab, "pad": 0, "dtype": "bf16", "temperature": 2.0, "top": 32,
            "ragged_top": False, "soft_weight": 0.5, "label_weight": 0.5, "left_out": 0.0, "train": True}
    case.update(options)
    return case


def _recur(name, batch, steps, width, **options):
    case = {"name": name, "kind": "recur", "batch": batch, "steps": steps, "width": width, "dtype": "bf16", "time_major": False,
            "out_gate": True, "lengths": False, "resets": False, "h0": True, "train": False}
    case.update(options)
    return case


def listed():
    return [
        # the next token of one stream: the recurrent model's vocabulary of 10000 words, with a few alternatives to show
        _score("score_one_token", 1, 10_000, dtype="f32", top=5),
        # one decoding step of a batch over a large vocabulary, sharpened, with the alternatives an API returns
        _score("score_decode_batch", 48, 131_072, temperature=0.8, top=20),
        # scoring whole texts: a vocabulary of odd size (rows start at odd places), one row in ten is a prompt or padding
        _score("score_texts", 6_001, 50_257, top=8, left_out=0.1),
        # a policy step: log probabilities and entropy, then the gradient of both
        _score("score_policy_step", 4_096, 32_000, train=True),
        # distillation of the recurrent model: 20 streams of 35 steps over 10000 words
        _distill("distill_lstm_step", 700, 10_000, dtype="f32", top=16),
        # a few long rows: the step of a small micro-batch over a large vocabulary, soft targets alone
        _distill("distill_few_rows", 24, 131_072, dtype="f32", top=128, temperature=1.0, soft_weight=1.0, label_weight=0.0),
        # odd vocabulary padded to a multiple of 64, teachers that kept fewer entries where they were sure, no temperature
        _distill("distill_padded_vocab", 2_048, 50_257, pad=47, top=64, ragged_top=True, temperature=1.0),
        # a large batch of tokens
        _distill("distill_large", 8_192, 32_000),
        # one decoding step of 64 streams: one token each, state in, state out
        _recur("recur_one_step", 64, 1, 1_500),
        # truncated back-propagation on the recurrent model: 20 streams of 35 steps, 1500 units, time first
        _recur("recur_lstm_step", 20, 35, 1_500, dtype="f32", time_major=True, train=True),
        # reading one long prompt
        _recur("recur_prompt", 1, 32_768, 1_500),
        # training on long rows into which several texts are packed: the state starts anew at each
        _recur("recur_packed_training", 8, 4_096, 2_048, resets=True, h0=False, train=True),
    ]


_LARGEST = 1_050_000_000   # bytes of the largest listed cases


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(["score", "score", "distill", "distill", "recur", "recur"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    train = rng.random() < 0.5
    if kind == "recur":
        batch, width = _log_uniform(rng, 1, 128), _log_uniform(rng, 64, 4_096)
        steps = 1 if rng.random() < 0.15 else _log_uniform(rng, 2, 32_768)
        case = _recur("", batch, steps, width, dtype=dtype, time_major=rng.random() < 0.3, out_gate=rng.random() < 0.7,
                      lengths=rng.random() < 0.3, resets=rng.random() < 0.3, h0=rng.random() < 0.5, train=train)
        size = "steps"
    else:
        rows, vocab = _log_uniform(rng, 1, 16_384), _log_uniform(rng, 1_000, 200_000)
        pad = rng.choice([0, 0, -vocab % 64])
        temperature = rng.choice([1.0, 1.0, 0.7, 2.0, 4.0])
        if kind == "score":
            case = _score("", rows, vocab, pad=pad, dtype=dtype, temperature=temperature, top=rng.choice([0, 1, 5, 20, 64]),
                          left_out=rng.choice([0.0, 0.3]), banned=rng.choice([0.0, 0.0, 0.5]), train=train)
        else:
            case = _distill("", rows, vocab, pad=pad, dtype=dtype, temperature=temperature, top=_log_uniform(rng, 1, 128),
                            ragged_top=rng.random() < 0.5, label_weight=rng.choice([0.0, 0.5]), left_out=rng.choice([0.0, 0.3]),
                            train=train)
        size = "rows"
    del case["name"]
    # the same bytes and, for the alternatives' sake, no more elements than the largest listed case has
    elements = case["batch"] * case["steps"] * case["width"] if kind == "recur" else case["rows"] * case["vocab"]
    most = min(_LARGEST / work(case)["bytes"], 67_000_000 / elements if kind == "recur" else 260_000_000 / elements)
    if most < 1.0:
        case[size] = max(1, int(case[size] * most))
    return case


def work(case):
    s = _SIZE[case["dtype"]]
    if case["kind"] == "recur":
        n, states = case["batch"] * case["steps"] * case["width"], case["batch"] * case["width"]
        tensors = (4 if case["out_gate"] else 3) + ((4 if case["out_gate"] else 3) if case["train"] else 0)
        extra = 4 * states * ((2 if case["h0"] else 1) + (2 if case["train"] else 0))
        extra += case["batch"] * case["steps"] if case["resets"] else 0
        # two sigmoids, the step and the product; backward the two scans, and three gradients
        return {"bytes": float(n * s * tensors + extra), "flops": float(n * (12 + (24 if case["train"] else 0)))}
    rows, n = case["rows"], case["rows"] * case["vocab"]
    if case["kind"] == "score":
        extra = rows * (4 + 4 + 4 + 8 * case["top"] + (8 if case["train"] else 0))
        return {"bytes": float(n * s * (2 if case["train"] else 1) + extra), "flops": float(n * (5 + (8 if case["train"] else 0)))}
    extra = rows * (8 * case["top"] + 8 + (4 if case["train"] else 0))
    return {"bytes": float(n * s * (2 if case["train"] else 1) + extra), "flops": float(n * (8 + (6 if case["train"] else 0)))}


# ------------------------------------------------------------------------------------------------ inputs

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _vocabulary_inputs(case, seed):
    """Logits of a language model: words of different frequency, a spread, and a clear favourite in half of the rows."""
    g, dev = _generator(seed), "cuda"
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    z = torch.randn(rows, vocab, generator=g, device=dev) * 2.0
    z += torch.randn(vocab, generator=g, device=dev)
    rows_at = torch.arange(rows, device=dev)
    favourite = torch.randint(0, vocab, (rows,), generator=g, device=dev)
    z[rows_at, favourite] += 14.0 * (torch.rand(rows, generator=g, device=dev) < 0.5)
    targets = torch.randint(0, vocab, (rows,), generator=g, device=dev)
    targets = torch.where(torch.rand(rows, generator=g, device=dev) < 0.5, favourite, targets)
    if case.get("banned"):
        z.masked_fill_(torch.rand(rows, vocab, generator=g, device=dev) < case["banned"], -math.inf)
        z[rows_at, targets] = 3.0
    if case["left_out"]:
        targets = torch.where(torch.rand(rows, generator=g, device=dev) < case["left_out"], torch.full_like(targets, -1), targets)
    buffer = torch.full((rows, vocab + case["pad"]), math.nan, dtype=_DTYPES[case["dtype"]], device=dev)
    buffer[:, :vocab] = z
    state = {"case": case, "logits": buffer[:, :vocab], "targets": targets.to(torch.int32)}
    if case["kind"] == "distill":
        z += torch.randn(rows, vocab, generator=g, device=dev) * 0.7
        value, index = torch.topk(z, top, dim=1)
        index = index.to(torch.int32)
        if case["ragged_top"]:
            kept = torch.randint(1, top + 1, (rows, 1), generator=g, device=dev)
            gone = torch.arange(top, device=dev) >= kept
            index.masked_fill_(gone, -1)
            value.masked_fill_(gone, 0.0)
        state.update(teacher_idx=index, teacher_logits=value.contiguous(), grad_loss=torch.rand(rows, generator=g, device=dev) + 0.5)
    elif case["train"]:
        state.update(grad_logprob=torch.randn(rows, generator=g, device=dev), grad_entropy=torch.randn(rows, generator=g, device=dev) * 0.1)
    return state


def _sequence_inputs(case, seed):
    """One projection's output, [.., 3 width] (or 2): inputs, gates that remember for a few to some hundred steps, output gates."""
    g, dev, dtype = _generator(seed), "cuda", _DTYPES[case["dtype"]]
    batch, steps, width = case["batch"], case["steps"], case["width"]
    parts = 3 if case["out_gate"] else 2
    lead = (steps, batch) if case["time_major"] else (batch, steps)

    def batch_first(t):
        return t.transpose(0, 1) if case["time_major"] else t

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=dev)

    projected = torch.empty(*lead, parts * width, dtype=dtype, device=dev)
    projected[..., :width] = normal(*lead, width)
    projected[..., width:2 * width] = normal(*lead, width) + (1.0 + 3.0 * torch.rand(width, generator=g, device=dev))
    if parts == 3:
        projected[..., 2 * width:] = normal(*lead, width)
    state = {"case": case, "projected": batch_first(projected), "lengths": None, "resets": None,
             "h0": normal(batch, width) if case["h0"] else None}
    if case["lengths"]:
        state["lengths"] = torch.randint(0, steps + 1, (batch,), generator=g, device=dev).to(torch.int32)
    if case["resets"]:
        state["resets"] = (torch.rand(batch, steps, generator=g, device=dev) < 1.0 / 300.0).to(torch.uint8)
    if case["train"]:
        state["dy"] = batch_first(normal(*lead, width).to(dtype))
        state["dh_last"] = normal(batch, width)
    return state


def _thirds(projected, width):
    """Inputs, gates and output gates (or None) of one projection's output."""
    return projected[..., :width], projected[..., width:2 * width], projected[..., 2 * width:] if projected.shape[-1] > 2 * width else None


_handle = []


def _context(rgc):
    """The program's one context (made at the first call)."""
    if not _handle:
        _handle.append(rgc.Context(1 << 16, 1))
    return _handle[0]


def prepare(case, seed):
    state = _sequence_inputs(case, seed) if case["kind"] == "recur" else _vocabulary_inputs(case, seed)
    if not own:
        return state
    # what a program keeps: the context, the output buffers, and the call's descriptor over both
    import paper_1808_04357_amd as rgc
    dev = "cuda"
    state["rgc"], state["ctx"], state["stream"] = rgc, _context(rgc), torch.cuda.current_stream()

    def f32(*shape):
        return torch.empty(*shape, dtype=torch.float32, device=dev)

    if case["kind"] == "recur":
        batch, steps, width = case["batch"], case["steps"], case["width"]
        x, gate, out_gate = _thirds(state["projected"], width)
        lead = (steps, batch) if case["time_major"] else (batch, steps)

        def like(parts):
            t = torch.empty(*lead, parts * width, dtype=x.dtype, device=dev)
            return t.transpose(0, 1) if case["time_major"] else t

        state["y"], state["h_last"] = like(1), f32(batch, width)
        kept = f32(batch, -(-steps // _STATE_STEPS), width) if case["train"] else None
        state["call"] = rgc.Recurrence(x, gate, state["y"], out_gate=out_gate, lengths=state["lengths"], resets=state["resets"],
                                       h0=state["h0"], h_last=state["h_last"], states=kept)
        if case["train"]:
            state["dprojected"], state["dh0"] = like(state["projected"].shape[-1] // width), f32(batch, width)
            dx, dgate, dout_gate = _thirds(state["dprojected"], width)
            state["grads"] = rgc.RecurrenceGrads(state["call"], state["dy"], dx, dgate, dout_gate=dout_gate,
                                                 dh_last=state["dh_last"], dh0=state["dh0"])
        return state
    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    if case["train"]:
        state["grad_logits"] = torch.empty(rows, vocab + case["pad"], dtype=state["logits"].dtype, device=dev)[:, :vocab]
    if case["kind"] == "score":
        state["logprob"], state["entropy"] = f32(rows), f32(rows)
        state["top_idx"] = torch.empty(rows, top, dtype=torch.int32, device=dev) if top else None
        state["top_logprob"] = f32(rows, top) if top else None
        state["call"] = rgc.TokenScores(state["logits"], state["targets"], logprob=state["logprob"], entropy=state["entropy"],
                                        top_idx=state["top_idx"], top_logprob=state["top_logprob"],
                                        stats=f32(rows, 2) if case["train"] else None, temperature=case["temperature"])
    else:
        state["loss"] = f32(rows)
        state["call"] = rgc.Distillation(state["logits"], state["teacher_idx"], state["teacher_logits"], targets=state["targets"],
                                         loss=state["loss"], grad_loss=state["grad_loss"] if case["train"] else None,
                                         grad_logits=state["grad_logits"] if case["train"] else None,
                                         temperature=case["temperature"], soft_weight=case["soft_weight"],
                                         label_weight=case["label_weight"])
    return state


# ------------------------------------------------------------------------------------------------ the calls

def run(state):
    if own:
        return _call(state)
    return {"score": _plain_score, "distill": _plain_distill, "recur": _plain_recur}[state["case"]["kind"]](state)


def _call(state):
    rgc, case, ctx, stream = state["rgc"], state["case"], state["ctx"], state["stream"]
    if case["kind"] == "recur":
        rgc.rgc_gated_recurrence(ctx, state["call"], stream)
        out = {"y": state["y"], "h_last": state["h_last"]}
        if case["train"]:
            rgc.rgc_gated_recurrence_backward(ctx, state["call"], state["grads"], stream)
            out.update(dprojected=state["dprojected"], dh0=state["dh0"])
        return out
    if case["kind"] == "distill":
        rgc.rgc_distill_loss(ctx, state["call"], stream)
        return {"loss": state["loss"], "grad_logits": state["grad_logits"]} if case["train"] else {"loss": state["loss"]}
    rgc.rgc_token_logprobs(ctx, state["call"], stream)
    out = {"logprob": state["logprob"], "entropy": state["entropy"]}
    if case["top"]:
        out.update(top_idx=state["top_idx"], top_logprob=state["top_logprob"])
    if case["train"]:
        rgc.rgc_token_logprobs_backward(ctx, state["call"], state["grad_logits"], grad_logprob=state["grad_logprob"],
                                        grad_entropy=state["grad_entropy"], stream=stream)
        out["grad_logits"] = state["grad_logits"]
    return out


# ------------------------------------------------------------------------------------------------ the plain forms

def _log_softmax(z):
    """Rows' log probabilities and the sums' logarithms; -inf for a logit of -inf, in a row of nothing else too."""
    m = z.amax(dim=1, keepdim=True)
    d = z - torch.where(m == -math.inf, torch.zeros_like(m), m)
    return torch.where(d == -math.inf, d, d - d.exp().sum(dim=1, keepdim=True).log())


def _is_token(index, vocab):
    return (index >= 0) & (index < vocab)


def _plain_score(state):
    case, temperature, top = state["case"], state["case"]["temperature"], state["case"]["top"]
    logits, vocab = state["logits"].float(), state["case"]["vocab"]
    there = _is_token(state["targets"], vocab)
    target = state["targets"].clamp(0, vocab - 1).long()[:, None]
    logp = _log_softmax(logits / temperature)
    p = logp.exp()
    entropy = -torch.where(p == 0, torch.zeros_like(p), p * logp).sum(dim=1)
    none = torch.zeros_like(entropy)
    out = {"logprob": torch.where(there, logp.gather(1, target)[:, 0], none), "entropy": torch.where(there, entropy, none)}
    if top:
        # one whole number a logit, larger for a larger logit and, where two are equal, for the lower index
        bits = (logits + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits)
        order = torch.where(torch.isnan(logits), torch.full_like(order, 0x7FFFFFFF), order)
        key = (order.long() << 32) + torch.arange(vocab - 1, -1, -1, device=order.device)
        index = vocab - 1 - (torch.topk(key, top, dim=1).values & 0xFFFFFFFF)
        at_top = logp.gather(1, index)
        out["top_idx"] = torch.where(there[:, None], index, torch.full_like(index, -1)).to(torch.int32)
        out["top_logprob"] = torch.where(there[:, None], at_top, torch.full_like(at_top, -math.inf))
    if case["train"]:
        dlogp = -state["grad_logprob"][:, None] * p
        dlogp.scatter_add_(1, target, state["grad_logprob"][:, None])
        spread = torch.where(p == 0, torch.zeros_like(p), p * (logp + entropy[:, None]))
        grad = (dlogp - state["grad_entropy"][:, None] * spread) / temperature
        grad = torch.where((there & (logits.amax(dim=1) != -math.inf))[:, None], grad, torch.zeros_like(grad))
        out["grad_logits"] = grad.to(state["logits"].dtype)
    return out


def _plain_distill(state):
    case, temperature, vocab = state["case"], state["case"]["temperature"], state["case"]["vocab"]
    z, index = state["logits"].float(), state["teacher_idx"]
    known = _is_token(index, vocab)
    index = index.clamp(0, vocab - 1).long()
    logq = _log_softmax(torch.where(known, state["teacher_logits"] / temperature, torch.full_like(state["teacher_logits"], -math.inf)))
    q = logq.exp()
    soft_weight = case["soft_weight"] * (q.sum(dim=1, keepdim=True) > 0)
    soft_logp = _log_softmax(z / temperature)
    soft = torch.where(q > 0, q * (logq - soft_logp.gather(1, index)), torch.zeros_like(q)).sum(dim=1) * temperature ** 2
    target = state["targets"].clamp(0, vocab - 1).long()[:, None]
    label_weight = case["label_weight"] * _is_token(state["targets"], vocab)[:, None]
    logp = _log_softmax(z)
    label = torch.where(label_weight[:, 0] > 0, -logp.gather(1, target)[:, 0], torch.zeros_like(soft))
    out = {"loss": soft_weight[:, 0] * soft + label_weight[:, 0] * label}
    if case["train"]:
        grad = soft_weight * temperature * soft_logp.exp().scatter_add(1, index, -q) + label_weight * logp.exp()
        grad.scatter_add_(1, target, -label_weight)
        out["grad_logits"] = (state["grad_loss"][:, None] * grad).to(state["logits"].dtype)
    return out


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1, from h = 0: every pass joins stretches twice as long.  (Overwrites both.)"""
    step = 1
    while step < b.shape[1]:
        b[:, step:] += a[:, step:] * b[:, :-step]
        a[:, step:] = a[:, step:] * a[:, :-step]
        step *= 2
    return b


def _plain_recur(state):
    case, width, steps = state["case"], state["case"]["width"], state["case"]["steps"]
    x, gate, out_gate = (None if t is None else t.float() for t in _thirds(state["projected"], width))
    there = torch.ones_like(x[..., :1], dtype=torch.bool)
    if case["lengths"]:
        there = (torch.arange(steps, device=x.device) < state["lengths"][:, None])[..., None]
        x, gate = x.where(there, torch.zeros_like(x)), gate.where(there, torch.zeros_like(gate))
    keep, take = torch.sigmoid(gate), torch.sigmoid(-gate)
    shut = torch.ones_like(keep) if out_gate is None else torch.sigmoid(out_gate)
    a = keep if not case["resets"] else keep * (state["resets"] == 0)[..., None]
    a = a.where(there, torch.ones_like(a))                       # behind a row's end the state stays as it is
    b = (take * x).where(there, torch.zeros_like(x))
    h0 = state["h0"] if case["h0"] else torch.zeros_like(x[:, 0])
    b[:, 0] += a[:, 0] * h0
    h = _scan(a.clone(), b)
    out = {"y": (shut * h).where(there, torch.zeros_like(h)).to(state["projected"].dtype), "h_last": h[:, -1].clone()}
    if case["train"]:
        dy = state["dy"].float().where(there, torch.zeros_like(x))
        e = dy * shut
        e[:, -1] += state["dh_last"]
        after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], dim=1)
        d = _scan(after.flip(1), e.flip(1)).flip(1)
        before = torch.cat([h0[:, None], h[:, :-1]], dim=1)
        if case["resets"]:
            before = before * (state["resets"] == 0)[..., None]
        parts = [d * take, d * (before - x) * keep * take] + ([] if out_gate is None else [dy * h * shut * torch.sigmoid(-out_gate)])
        out["dprojected"] = torch.cat([t.where(there, torch.zeros_like(t)) for t in parts], dim=2).to(state["projected"].dtype)
        out["dh0"] = a[:, 0] * d[:, 0]
    return out


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    if case["kind"] == "recur":
        return _exact_recur(case, _sequence_inputs(case, seed))
    state = _vocabulary_inputs(case, seed)
    rows_of = {k: v for k, v in state.items() if torch.is_tensor(v)}
    few = max(1, 30_000_000 // case["vocab"])
    parts = [(_exact_score if case["kind"] == "score" else _exact_distill)(case, {k: v[i:i + few] for k, v in rows_of.items()})
             for i in range(0, case["rows"], few)]
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _exact_score(case, t):
    z = t["logits"].double()
    target = t["targets"].long()
    left_out = (target < 0) | (target >= case["vocab"])
    at = target.masked_fill(left_out, 0).unsqueeze(1)
    logp = (z / case["temperature"]).log_softmax(dim=1)
    p = logp.exp()
    entropy = torch.special.entr(p).sum(dim=1)
    out = {"logprob": logp.gather(1, at).squeeze(1).masked_fill(left_out, 0.0), "entropy": entropy.masked_fill(left_out, 0.0)}
    if case["top"]:
        index = z.sort(dim=1, descending=True, stable=True).indices[:, :case["top"]]
        out["top_idx"] = index.masked_fill(left_out[:, None], -1).to(torch.int32)
        out["top_logprob"] = logp.gather(1, index).masked_fill(left_out[:, None], -math.inf)
    if case["train"]:
        g, h = t["grad_logprob"].double()[:, None], t["grad_entropy"].double()[:, None]
        chosen = torch.zeros_like(p).scatter_(1, at, 1.0)
        grad = g * (chosen - p) + h * (torch.special.entr(p) - p * entropy[:, None])
        out["grad_logits"] = (grad / case["temperature"]).masked_fill(left_out[:, None], 0.0)
    return out


def _exact_distill(case, t):
    z, heat = t["logits"].double(), case["temperature"]
    index = t["teacher_idx"].long()
    unknown = (index < 0) | (index >= case["vocab"])
    index = index.masked_fill(unknown, 0)
    q = (t["teacher_logits"].double() / heat).masked_fill(unknown, -math.inf).softmax(dim=1)
    warm = (z / heat).log_softmax(dim=1)
    divergence = (torch.special.xlogy(q, q) - q * warm.gather(1, index)).sum(dim=1)
    target = t["targets"].long()
    left_out = (target < 0) | (target >= case["vocab"])
    at = target.masked_fill(left_out, 0).unsqueeze(1)
    cold = z.log_softmax(dim=1)
    weight = torch.where(left_out, 0.0, case["label_weight"]).double().unsqueeze(1)
    out = {"loss": case["soft_weight"] * heat * heat * divergence - weight[:, 0] * cold.gather(1, at)[:, 0]}
    if case["train"]:
        teacher = torch.zeros_like(z).scatter_add_(1, index, q)
        label = torch.zeros_like(z).scatter_(1, at, 1.0)
        grad = case["soft_weight"] * heat * (warm.exp() - teacher) + weight * (cold.exp() - label)
        out["grad_logits"] = t["grad_loss"].double()[:, None] * grad
    return out


def _exact_recur(case, state):
    """Step by step, as the formula stands."""
    width, steps, batch = case["width"], case["steps"], case["batch"]
    x, gate, out_gate = (None if t is None else t.double() for t in _thirds(state["projected"], width))
    keep = 1.0 / (1.0 + (-gate).exp())
    take = 1.0 / (1.0 + gate.exp())
    opened = torch.ones_like(keep) if out_gate is None else 1.0 / (1.0 + (-out_gate).exp())
    there = torch.ones(batch, steps, 1, dtype=torch.float64, device=x.device)
    if case["lengths"]:
        there = (torch.arange(steps, device=x.device)[None] < state["lengths"][:, None]).double()[..., None]
    carried = keep if not case["resets"] else keep * (1.0 - state["resets"].double())[..., None]
    carried = carried * there + (1.0 - there)
    h = torch.empty(batch, steps + 1, width, dtype=torch.float64, device=x.device)
    h[:, 0] = state["h0"].double() if case["h0"] else 0.0
    fed = take * x * there
    for t in range(steps):
        torch.addcmul(fed[:, t], carried[:, t], h[:, t], out=h[:, t + 1])
    out = {"y": opened * h[:, 1:] * there, "h_last": h[:, -1].clone()}
    if case["train"]:
        dy = state["dy"].double() * there
        d = dy * opened
        d[:, -1] += state["dh_last"].double()
        for t in range(steps - 2, -1, -1):
            d[:, t].addcmul_(carried[:, t + 1], d[:, t + 1])
        before = h[:, :-1]
        if case["resets"]:
            before = before * (1.0 - state["resets"].double())[..., None]
        parts = [d * take * there, d * (before - x) * keep * take * there]
        if out_gate is not None:
            parts.append(dy * h[:, 1:] * opened * (1.0 - opened))
        out["dprojected"] = torch.cat(parts, dim=2)
        out["dh0"] = carried[:, 0] * d[:, 0]
    return out
