"""A small recurrent language model, trained by distillation on several (virtual) data-parallel workers that exchange compressed gradients.

The operators together, as a program uses them: a teacher scores its tokens (rgc_gated_recurrence, rgc_token_logprobs: its top alternatives), every
worker's student learns from them (rgc_gated_recurrence, rgc_distill_loss, rgc_gated_recurrence_backward), the gradients are compressed
(rgc_compress_layers), the messages of all workers added up (rgc_decompress_accumulate) and applied; at last the student continues a text one token at
a time, its state updated in place, with the log probability of what it says and what else it might have said.

    python examples/recurrent_lm.py [--steps 150] [--workers 4]
"""
from __future__ import annotations

import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_1808_04357_amd as rgc  # noqa: E402


class Model:
    """Embedding, one gated recurrent layer (input, gate and output gate from one product), output product; float32."""

    def __init__(self, vocab: int, width: int, seed: int, scale: float = 1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def weight(*shape, spread):
            return torch.randn(*shape, generator=g, device="cuda") * spread

        self.vocab, self.width = vocab, width
        self.parameters = {"embedding": weight(vocab, width, spread=1.0), "inner": weight(width, 3 * width, spread=scale * width ** -0.5),
                           "output": weight(width, vocab, spread=2.0 * scale * width ** -0.5)}


class Run:
    """The buffers and descriptors of a model's passes over [batch, steps] tokens, made once."""

    def __init__(self, model: Model, batch: int, steps: int):
        self.model, self.batch, self.steps = model, batch, steps
        width = model.width

        def empty(*shape):
            return torch.empty(*shape, device="cuda")

        self.inner, self.dinner = empty(batch, steps, 3 * width), empty(batch, steps, 3 * width)
        self.y, self.dy = empty(batch, steps, width), empty(batch, steps, width)
        self.h = torch.zeros(batch, width, device="cuda")
        states = empty(batch, -(-steps // rgc.RGC_RECURRENCE_CHUNK), width)
        x, gate, out_gate = self.inner.split(width, dim=2)
        dx, dgate, dout_gate = self.dinner.split(width, dim=2)
        self.recurrence = rgc.Recurrence(x, gate, self.y, out_gate=out_gate, h_last=empty(batch, width), states=states)
        self.grads = rgc.RecurrenceGrads(self.recurrence, self.dy, dx, dgate, dout_gate=dout_gate)
        # one token at a time: the same weights, the state in place
        self.one = rgc.Recurrence(x[:, :1], gate[:, :1], self.y[:, :1], out_gate=out_gate[:, :1], h0=self.h, h_last=self.h)
        self.logits = empty(batch * steps, model.vocab)
        self.dlogits = torch.empty_like(self.logits)

    def forward(self, ctx, tokens, stream):
        p = self.model.parameters
        torch.matmul(p["embedding"][tokens], p["inner"], out=self.inner)
        rgc.rgc_gated_recurrence(ctx, self.recurrence, stream)
        torch.matmul(self.y.view(-1, self.model.width), p["output"], out=self.logits)

    def backward(self, ctx, tokens, stream):
        """Gradients of the parameters, from self.dlogits."""
        p, width = self.model.parameters, self.model.width
        torch.matmul(self.dlogits, p["output"].t(), out=self.dy.view(-1, width))
        rgc.rgc_gated_recurrence_backward(ctx, self.recurrence, self.grads, stream)
        dinner, x = self.dinner.view(-1, 3 * width), p["embedding"][tokens].view(-1, width)
        embedding = torch.zeros_like(p["embedding"])
        embedding.index_add_(0, tokens.reshape(-1), dinner @ p["inner"].t())
        return {"embedding": embedding, "inner": x.t() @ dinner, "output": self.y.view(-1, width).t() @ self.dlogits}


class Teacher:
    """Its log probabilities of the next tokens: the top ones, with their indices."""

    def __init__(self, model: Model, batch: int, steps: int, top: int):
        self.run = Run(model, batch, steps)
        rows = batch * steps
        self.index = torch.empty(rows, top, dtype=torch.int32, device="cuda")
        self.logprob = torch.empty(rows, top, device="cuda")
        self.scores = rgc.TokenScores(self.run.logits, top_idx=self.index, top_logprob=self.logprob)

    def __call__(self, ctx, tokens, stream):
        self.run.forward(ctx, tokens, stream)
        rgc.rgc_token_logprobs(ctx, self.scores, stream)


class Worker:
    """One data-parallel worker: its residuals, its messages, its context (threshold hints are a worker's own)."""

    def __init__(self, model: Model, teacher: Teacher, batch: int, steps: int, density_ppm: int):
        self.run, self.teacher = Run(model, batch, steps), teacher
        rows = batch * steps
        self.targets = torch.empty(rows, dtype=torch.int32, device="cuda")
        self.loss = torch.empty(rows, device="cuda")
        self.weight = torch.full((rows,), 1.0 / rows, device="cuda")
        self.distillation = rgc.Distillation(self.run.logits, teacher.index, teacher.logprob, targets=self.targets, loss=self.loss,
                                             grad_loss=self.weight, grad_logits=self.run.dlogits, temperature=2.0, soft_weight=0.7,
                                             label_weight=0.3)
        sizes = [p.numel() for p in model.parameters.values()]
        self.ctx = rgc.Context(sum(sizes), len(sizes))
        self.gradients = [torch.empty(n, device="cuda") for n in sizes]
        self.residuals = [torch.zeros(n, device="cuda") for n in sizes]
        self.velocities = [torch.zeros(n, device="cuda") for n in sizes]
        ks = [rgc.rgc_k_for_density(n, density_ppm) for n in sizes]
        self.index = [torch.empty(k, dtype=torch.int32, device="cuda") for k in ks]
        self.value = [torch.empty(k, device="cuda") for k in ks]
        self.count = torch.empty(len(ks), dtype=torch.int32, device="cuda")
        self.layers = rgc.LayerList(self.gradients, self.residuals, ks, self.index, self.value, self.count, self.velocities)

    def learn(self, tokens, following, stream):
        """Loss and gradients of the student on these tokens; `following`: the tokens after them, negative where there is none."""
        self.teacher(self.ctx, tokens, stream)
        self.run.forward(self.ctx, tokens, stream)
        self.targets.copy_(following.reshape(-1))
        rgc.rgc_distill_loss(self.ctx, self.distillation, stream)
        return self.run.backward(self.ctx, tokens, stream)

    def compress(self, gradients, momentum, stream):
        for flat, g in zip(self.gradients, gradients.values()):
            flat.copy_(g.reshape(-1))
        rgc.rgc_compress_layers(self.ctx, self.layers, momentum, 0, stream)


def train(steps=150, workers=4, vocab=2_000, width=192, batch=4, length=48, top=16, density_ppm=100_000, rate=5.0, texts=2, seed=1):
    """Losses by step (mean over workers), and the student."""
    stream = torch.cuda.current_stream()
    teacher, student = Model(vocab, width, seed, scale=1.5), Model(vocab, width, seed + 1)
    team = [Worker(student, Teacher(teacher, batch, length, top), batch, length, density_ppm) for _ in range(workers)]
    update = [torch.empty(p.numel(), device="cuda") for p in student.parameters.values()]
    messages = rgc.MessageList([w.index for w in team], [w.value for w in team], update)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    corpus = torch.randint(0, vocab, (texts, workers, batch, length + 1), generator=g, device="cuda")      # every worker's share of it
    losses = []
    for step in range(steps):
        for worker, text in zip(team, corpus[step % texts]):
            worker.compress(worker.learn(text[:, :-1], text[:, 1:], stream), 0.9, stream)
        rgc.rgc_decompress_accumulate(team[0].ctx, messages, 1.0 / workers, rgc.RGC_OVERWRITE, stream)
        for p, u in zip(student.parameters.values(), update):
            p.view(-1).sub_(u, alpha=rate)
        losses.append(float(torch.stack([w.loss.mean() for w in team]).mean()))
    for worker in team:
        worker.ctx.close()
    return losses, student


def continue_text(student, tokens=12, top=3):
    """Greedy, one token at a time: [(token, its log probability, entropy, top alternatives)]."""
    stream, ctx = torch.cuda.current_stream(), rgc.Context(1, 1)
    run, p, width = Run(student, 1, 1), student.parameters, student.width
    target, logprob, entropy = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty(1, device="cuda"), torch.empty(1, device="cuda")
    index, value = torch.empty(1, top, dtype=torch.int32, device="cuda"), torch.empty(1, top, device="cuda")
    scores = rgc.TokenScores(run.logits, top_idx=index, top_logprob=value, entropy=entropy)
    said = rgc.TokenScores(run.logits, target, logprob=logprob)
    token, out = 0, []
    for _ in range(tokens):
        torch.matmul(p["embedding"][token:token + 1], p["inner"], out=run.inner.view(1, -1))
        rgc.rgc_gated_recurrence(ctx, run.one, stream)
        torch.matmul(run.y.view(-1, width), p["output"], out=run.logits)
        rgc.rgc_token_logprobs(ctx, scores, stream)
        target.copy_(index[0, :1])
        rgc.rgc_token_logprobs(ctx, said, stream)
        token = int(index[0, 0])
        out.append((token, float(logprob), float(entropy), list(zip(index[0].tolist(), value[0].tolist()))))
    torch.cuda.synchronize()
    ctx.close()
    return out


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=150)
    parser.add_argument("--workers", type=int, default=4)
    args = parser.parse_args()
    losses, student = train(args.steps, args.workers)
    for step in range(0, args.steps, 25):
        print("step %3d  loss %.4f" % (step, losses[step]))
    print("step %3d  loss %.4f" % (args.steps - 1, losses[-1]))
    for token, logprob, entropy, others in continue_text(student):
        print("token %5d  log p %.3f  entropy %.3f  top %s" % (token, logprob, entropy, ", ".join("%d (%.3f)" % o for o in others)))


if __name__ == "__main__":
    main()
