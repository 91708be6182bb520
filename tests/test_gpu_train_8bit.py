"""The 8-bit layer's operators together with the optimizer's step, as examples/train_8bit.py uses them: gradients of the whole network
against torch's of the same network in fp32, and a training run against AdamW in fp32."""
import importlib.util
import os

import pytest
import torch

import paper_2604_06836_amd as stq

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("train_8bit", os.path.join(ROOT, "examples", "train_8bit.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def norm(x, w, eps):
    return x * torch.rsqrt(x.square().mean(1, keepdim=True) + eps) * w


def network(p, x, eps):
    for b in p["blocks"]:
        both = norm(x, b["norm"], eps) @ b["gate_up"].t()
        gate, up = both.chunk(2, 1)
        x = x + (gate * torch.sigmoid(gate) * up) @ b["down"].t()
    return norm(x, p["norm"], eps) @ p["head"].t()


def tensors(p):
    return [t for b in p["blocks"] for t in (b["norm"], b["gate_up"], b["down"])] + [p["norm"], p["head"]]


def test_gradients_of_the_network(example):
    """8-bit operands are off by up to half a code of 127 of their row's largest value, about 1 % of the typical one, and there are
    five products one behind the other: outputs and gradients agree with fp32's to a few per cent in the 2-norm."""
    tokens, d, f, outputs = 300, 256, 512, 16
    ctx = stq.Context(0, 16)
    p = example.make_params(d, f, outputs, 2, seed=3)
    net = example.Net(ctx, p, tokens)
    x, y = next(example.batches(1, tokens, d, outputs, seed=4))
    out = net.forward(x)
    diff = out - y
    net.backward((2 * diff / diff.numel()).bfloat16())
    for t in tensors(p):
        t.requires_grad_(True)
    want = network(p, x.float(), example.EPS)
    assert ((out - want).norm() / want.norm()).item() < 0.05
    grads = torch.autograd.grad(want, tensors(p), 2 * diff / diff.numel())
    got = [g for b in net.blocks for g in (b.norm.grad, b.gate_up.grad, b.down.grad)] + [net.norm.grad, net.head.grad]
    for g, w in zip(got, grads):
        assert ((g.float() - w).norm() / w.norm()).item() < 0.08
    torch.cuda.synchronize()
    ctx.close()


def test_training_keeps_up_with_fp32(example):
    steps, tokens, d, f, outputs = 150, 512, 256, 512, 16
    losses = example.train(steps, tokens, d, f, outputs, 2, lr=1e-3)
    p = example.make_params(d, f, outputs, 2, seed=0)
    for t in tensors(p):
        t.requires_grad_(True)
    opt = torch.optim.AdamW(tensors(p), lr=1e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.0)
    reference = []
    for x, y in example.batches(steps, tokens, d, outputs, seed=1):
        loss = (network(p, x.float(), example.EPS) - y).square().mean()
        opt.zero_grad(set_to_none=True)
        loss.backward()
        opt.step()
        reference.append(loss.item())
    last, want = sum(losses[-20:]) / 20, sum(reference[-20:]) / 20
    assert all(l == l for l in losses)
    assert last < 0.6 * losses[0], (losses[0], last)
    assert last < 1.15 * want, (last, want)
