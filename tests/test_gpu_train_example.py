"""The example classifier: one step's gradients against torch's own gradients in
64 bits on the CPU, and a short training that learns."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location(
        "train_classifier", os.path.join(ROOT, "examples", "train_classifier.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_step_matches_torch(example):
    F = torch.nn.functional
    p = example.parameters()
    x, labels = example.images(16, torch.Generator().manual_seed(3))
    out, g, norm = example.step(p, x, labels, max_norm=float("inf"))
    q = {k: v.cpu().double().requires_grad_() for k, v in p.items()}
    a = F.max_pool2d(F.relu(F.conv2d(x.cpu().double(), q["w1"], q["b1"], padding=1)), 2)
    a = F.relu(F.conv2d(a, q["w2"], q["b2"], padding=1)).mean((2, 3))
    a = F.layer_norm(a, a.shape[1:], q["scale"], q["shift"], 1e-5)
    logp = F.log_softmax(F.conv2d(a[:, :, None, None], q["w3"], q["b3"])[:, :, 0, 0], 1)
    loss = -logp.gather(1, labels.cpu()[:, None]).mean()
    loss.backward()
    assert abs(float(-out.logp.mean()) - float(loss.detach())) < 1e-5
    total = sum(float((v.grad ** 2).sum()) for v in q.values()) ** 0.5
    assert abs(float(norm) / total - 1) < 1e-4
    for k in p:
        err = (g[k].cpu().double() - q[k].grad).norm() / q[k].grad.norm()
        assert float(err) < 1e-4, k
    _, clipped, _ = example.step(p, x, labels, max_norm=0.1 * total)
    size = sum(float((v.double() ** 2).sum()) for v in clipped.values()) ** 0.5
    assert abs(size / (0.1 * total) - 1) < 1e-4


def test_training_learns(example):
    losses = example.train(40, 32)
    assert losses[0] > 2.0 and sum(losses[-5:]) / 5 < 0.3 * losses[0]
