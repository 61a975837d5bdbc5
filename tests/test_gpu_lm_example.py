"""The example that runs the language-model operators together with the compression: its gradients against automatic differentiation
of the same model in 64 bits, its training, and its one-token-at-a-time form against the form over whole sequences."""
import importlib.util
import os

import numpy as np
import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    spec = importlib.util.spec_from_file_location("recurrent_lm", os.path.join(ROOT, "examples", "recurrent_lm.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def model64(parameters, tokens):
    """Logits in 64 bits on the CPU, step by step; differentiable."""
    import torch
    x = parameters["embedding"][tokens]
    width = x.shape[-1]
    inner = x @ parameters["inner"]
    value, keep, open_ = inner[..., :width], torch.sigmoid(inner[..., width:2 * width]), torch.sigmoid(inner[..., 2 * width:])
    h, ys = torch.zeros(x.shape[0], width, dtype=torch.float64), []
    for t in range(x.shape[1]):
        h = keep[:, t] * h + (1 - keep[:, t]) * value[:, t]
        ys.append(open_[:, t] * h)
    return torch.stack(ys, dim=1) @ parameters["output"]


def test_gradients_of_a_worker_are_those_of_the_loss(example):
    import torch
    vocab, width, batch, length = 301, 40, 3, 21
    teacher, student = example.Model(vocab, width, 5, 1.5), example.Model(vocab, width, 6)
    worker = example.Worker(student, example.Teacher(teacher, batch, length, 8), batch, length, 1000)
    g = torch.Generator(device="cuda").manual_seed(7)
    text = torch.randint(0, vocab, (batch, length + 1), generator=g, device="cuda")
    following = text[:, 1:].clone()
    following[1, 5:9] = -1                               # no labels there
    got = worker.learn(text[:, :-1], following, torch.cuda.current_stream())
    torch.cuda.synchronize()
    tokens, after = text[:, :-1].cpu(), following.cpu().reshape(-1)
    exact = {k: v.double().cpu() for k, v in teacher.parameters.items()}
    said = torch.log_softmax(model64(exact, tokens).reshape(-1, vocab), dim=1)
    index = worker.teacher.index.cpu().long()
    assert torch.equal(said.topk(8, dim=1).indices, index)
    # float32 products over 40 and 301 terms in front of the operators: a few 1e-6 of the values' size
    assert torch.allclose(said.gather(1, index).float(), worker.teacher.logprob.cpu(), atol=2e-5)
    own = {k: v.double().cpu().requires_grad_() for k, v in student.parameters.items()}
    z = model64(own, tokens).reshape(-1, vocab)
    q = torch.softmax(said.gather(1, index) / 2.0, dim=1)
    soft = 4.0 * (q * (q.log() - torch.log_softmax(z / 2.0, dim=1).gather(1, index))).sum(dim=1)
    label = torch.where(after < 0, 0.0, -torch.log_softmax(z, dim=1).gather(1, after.clamp(min=0)[:, None])[:, 0])
    loss = 0.7 * soft + 0.3 * label
    loss.mean().backward()
    assert torch.allclose(loss.detach().float(), worker.loss.cpu(), rtol=1e-4, atol=1e-4)
    for k in own:
        want, have = own[k].grad, got[k].double().cpu()
        assert float((have - want).norm() / want.norm()) < 1e-4, k
    worker.ctx.close()


def test_training_lowers_the_loss_and_the_student_speaks(example):
    losses, student = example.train(steps=100, workers=2, vocab=400, width=64, batch=4, length=24)
    assert all(np.isfinite(losses)) and np.mean(losses[-5:]) < 0.9 * np.mean(losses[:5]), losses
    said = example.continue_text(student, tokens=5)
    assert len(said) == 5
    for token, logprob, entropy, others in said:
        assert token == others[0][0] and abs(logprob - others[0][1]) < 1e-6 and entropy >= 0.0
        assert [v for _, v in others] == sorted((v for _, v in others), reverse=True)


def test_one_token_at_a_time_is_the_whole_sequence(example):
    import torch
    import paper_1808_04357_amd as rgc
    model = example.Model(211, 36, 9)
    ctx, stream = rgc.Context(1, 1), torch.cuda.current_stream()
    tokens = torch.randint(0, 211, (2, 17), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    whole, one = example.Run(model, 2, 17), example.Run(model, 2, 1)
    whole.forward(ctx, tokens, stream)
    for t in range(17):
        torch.matmul(model.parameters["embedding"][tokens[:, t:t + 1]], model.parameters["inner"], out=one.inner)
        rgc.rgc_gated_recurrence(ctx, one.one, stream)
        torch.cuda.synchronize()
        assert torch.allclose(one.y[:, 0], whole.y[:, t], rtol=1e-4, atol=1e-5), t
    ctx.close()
