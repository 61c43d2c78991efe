"""The operators of a local step together, as examples/distill_student.py uses them: gradients of the whole model against
64-bit differentiation, and training through Slim-DP rounds."""
import importlib.util
import os

import pytest
import torch

import _train_ref as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def student():
    spec = importlib.util.spec_from_file_location("distill_student", os.path.join(ROOT, "examples", "distill_student.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def reference(lay, flat, batch, idx, teacher, label, T, kd, ce):
    """The same model in 64 bits, differentiated by autograd."""
    flat = flat.double().requires_grad_(True)
    x = batch.double()

    def norm(v, gamma, beta):
        c = v - v.mean(1, keepdim=True)
        return c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * gamma + beta

    p = lambda name: lay.view(flat, name)                                         # noqa: E731
    for b in range(lay.blocks):
        h = R.act(norm(x, p(f"{b}.gamma"), p(f"{b}.beta")) @ p(f"{b}.w1").t() + p(f"{b}.b1"), "gelu")
        x = x + h @ p(f"{b}.w2").t() + p(f"{b}.b2")
    z = norm(x, p("gamma"), p("beta")) @ p("wv").t() + p("bv")
    q = torch.softmax(teacher.double() / T, 1)
    logp = torch.gather(torch.log_softmax(z / T, 1), 1, idx.long())
    loss = kd * T * T * (q * (torch.log(q) - logp)).sum(1) - ce * torch.gather(torch.log_softmax(z, 1), 1, label.long()[:, None])[:, 0]
    loss.mean().backward()
    return loss.detach(), flat.grad


# fp32: a few hundred roundings of 2^-24 on the way through a dozen operators; 16-bit types: each of the about 20 tensors between
# operators is rounded once, 2^-9 (2^-12) relative on average, and their errors add up like independent ones
@pytest.mark.parametrize("dtype,allowed", [(torch.float32, 2e-5), (torch.bfloat16, 20 ** 0.5 * 2 * 2.0 ** -8), (torch.float16, 20 ** 0.5 * 2 * 2.0 ** -11)])
def test_gradient_of_the_whole_model(student, dtype, allowed):
    lay = student.Layout(2, 96, 200, 333)
    flat = lay.init(3)
    flat.copy_(flat.to(dtype).float())                         # weights that the type holds
    g = R.gen(4)
    batch = torch.randn(70, 96, generator=g, device="cuda").to(dtype).float()
    idx, teacher, label = student.synthetic_teacher(lay, 5, 9)(batch)
    worker = student.Worker(lay, 70, dtype, 9)
    delta = torch.zeros(lay.n, device="cuda")
    scale = 1.0 if dtype != torch.float16 else 1024.0
    worker.row_weight.mul_(scale)                              # fp16's gradients would be subnormal
    loss = worker.step(flat, delta, batch, idx, teacher, label) / scale
    rl, rg = reference(lay, flat, batch, idx, teacher, label, 2.0, 0.9, 0.1)
    assert ((loss.double() * 70 - rl).norm() / rl.norm()).item() <= allowed
    for name, (start, shape) in lay.at.items():
        got, ref = lay.view(delta, name).double() / scale, lay.view(rg, name)
        assert ((got - ref).norm() / ref.norm()).item() <= allowed, name
    # a second step adds to the update
    twice = delta.clone()
    worker.step(flat, twice, batch, idx, teacher, label)
    assert torch.allclose(twice, 2 * delta, rtol=1e-5, atol=1e-12)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_training_through_rounds_lowers_the_loss(student, dtype):
    losses = student.train(rounds=30, dtype=dtype)
    assert all(torch.isfinite(torch.tensor(losses)))
    assert losses[-1] < 0.8 * losses[0]
