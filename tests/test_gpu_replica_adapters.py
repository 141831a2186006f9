"""The adapters' example: its gradient of all replicas against a differentiated model in 64 bits, its training and its generation."""
import os
import sys

import pytest

torch = pytest.importorskip("torch")
from paper_2509_03110_amd import ops  # noqa: E402

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
import replica_adapters as ra  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradient_against_64_bits():
    K, seqs, length, p, seed, step = 3, 2, 19, 0.25, 5, 11
    model = ra.Model(vocab=50, dim=40, rank=6, dtype=torch.float32)
    rows = torch.stack([model.start(k) for k in range(K)])
    rows[:, :model.d] += 0.1 * torch.randn(K, model.d, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV)
    tokens = ra.sequences(K, seqs, length, model.vocab, 0, DEV)
    grads = torch.full_like(rows, float("nan"))
    loss = model.gradient(rows, tokens, grads, p, seed, step)

    kept = ops.dropout(torch.ones(K, seqs * length, model.dim, device=DEV), p, seed, step).cpu().double() * (1 - p)
    kept = (kept > 0.5).double() / (1 - p)                  # 65536 p is whole: the scale is 1 / (1 - p)
    w = rows[:, :model.d].cpu().double().requires_grad_()
    E, W = model.E.cpu().double(), {n: m.cpu().double() for n, m in model.W.items()}
    want_loss = []
    for k in range(K):
        def adapted(name, inp):
            (a, sa), (b, sb) = model.place[name + "A"], model.place[name + "B"]
            A, B = w[k, a:a + sa[0] * sa[1]].view(sa), w[k, b:b + sb[0] * sb[1]].view(sb)
            return inp @ W[name].T + model.scale * (inp @ A.T) @ B.T
        e = E[tokens[k, :, :-1].reshape(-1).long().cpu()]
        f, x = adapted("f", e).view(seqs, length, -1), adapted("x", e).view(seqs, length, -1)
        h, hs = torch.zeros(seqs, model.dim, dtype=torch.float64), []
        for t in range(length):
            a = torch.sigmoid(f[:, t])
            h = a * h + (1 - a) * x[:, t]
            hs.append(h)
        r = e + kept[k] * torch.stack(hs, dim=1).reshape(seqs * length, -1)
        z = adapted("z", r)
        want_loss.append(torch.nn.functional.cross_entropy(z, tokens[k, :, 1:].reshape(-1).long().cpu()))
    torch.stack(want_loss).sum().backward()
    # fp32 values through four products, a recurrence and their gradients: some tens of roundings of 2^-24 of their size
    assert float((loss.cpu() - torch.stack(want_loss).detach()).abs().max()) < 1e-5
    got = grads[:, :model.d].cpu().double()
    for name, (at, shape) in model.place.items():
        part = slice(at, at + shape[0] * shape[1])
        want = w.grad[:, part]
        assert float((got[:, part] - want).norm() / want.norm()) < 1e-5, name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_and_generation(dtype):
    model = ra.Model(dtype=dtype)
    losses, y = ra.train(model, steps=40)
    assert bool(torch.isfinite(losses).all()) and losses.shape == (40, 4)
    assert float(losses[-5:].mean()) < float(losses[:5].mean()) - 0.5
    again, y2 = ra.train(model, steps=40)
    assert torch.equal(losses, again) and torch.equal(y, y2)                   # no sum's order changes
    made, entropy = model.generate(y, torch.tensor([0, 17, 40], dtype=torch.int32, device=DEV), 8)
    assert made.shape == (3, 8) and int(made.min()) >= 0 and int(made.max()) < model.vocab
    assert 0.0 < entropy < 4.2
