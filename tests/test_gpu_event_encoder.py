"""The example that runs the sequence operators together (examples/event_encoder.py): its gradients against 64-bit automatic differentiation of
the whole chain, its training, and serving one event at a time against whole sequences."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    import event_encoder
    return event_encoder


def test_gradients_of_the_chain(example):
    """fp32: rows of 192, at most 40 events a sequence; each of the chain's operators is within a few hundred units of 2^-24 of its operands
    (see their own tests), and three of them in turn within 1e-4 of the largest gradient."""
    enc = example.EventEncoder(50, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    for p in (enc.weight, enc.norm_bias, enc.bias):
        p += 0.3 * torch.randn(p.shape, generator=g, device="cuda")
    n = [7, 1, 40, 13]
    offsets = torch.tensor([0, 7, 8, 48, 61], device="cuda")
    ids = torch.randint(0, 50, (61,), generator=g, device="cuda")
    f = enc.forward(ids, offsets)
    dout = torch.randn(61, enc.heads, enc.dim, generator=g, device="cuda")
    got = enc.gradients(f, dout, offsets)
    leaves = [t.double().detach().requires_grad_() for t in (enc.tables.view(50, -1)[ids], enc.weight, enc.norm_bias, enc.bias)]
    x, w, b, table = leaves
    y = (x - x.mean(1, keepdim=True)) / (x.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt() * w + b
    q, k, v = y.view(-1, 3 * enc.heads, enc.dim).split(enc.heads, 1)
    outs, far = [], enc.bucket_map.numel() // 2
    for i, m in enumerate(n):
        s = slice(int(offsets[i]), int(offsets[i + 1]))
        d = torch.arange(m, device="cuda")[:, None] - torch.arange(m, device="cuda")
        score = torch.einsum("ihd,jhd->hij", q[s], k[s]) * enc.dim ** -0.5 + table[:, enc.bucket_map.long()[d.clamp(-far, far) + far]]
        outs.append(torch.einsum("hij,jhd->ihd", score.masked_fill(d < 0, -float("inf")).softmax(2), v[s]))
    out = torch.cat(outs)
    assert (f["out"].double() - out).abs().max() <= 1e-4 * out.abs().max()
    out.backward(dout.double())
    for a, leaf in zip(got, leaves):
        assert (a.double() - leaf.grad).abs().max() <= 1e-4 * leaf.grad.abs().max()


@pytest.mark.parametrize("io,apart", [("f32", 1e-5), ("bf16", 0.1)])
def test_training_and_serving(example, io, apart):
    losses, worst = example.main(["--steps", "25", "--users", "64", "--ids", "100", "--io", io])
    assert losses[-1] < 0.8 * losses[0]
    assert worst <= apart
