"""K replicas of low-rank adapters, held together by the sharpness-aware elastic step, on one frozen language model; then the
center's adapters generate.

The model: a token's embedding e gives a gate f and an input x through two adapted matrices; h is their gated recurrence along the
sequence; r = e + dropout(h); an adapted matrix makes the logits.  A replica's parameters are its six adapter factors, one row
of a [K, d] array: the adapter calls read them, and write their gradients, as parts of that row, and the update takes the same
rows.  All K replicas go through the frozen matrices together, as K segments of one batch.

    python examples/replica_adapters.py [--steps 60] [--dtype bf16]
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_03110_amd import lsam, ops  # noqa: E402


class Model:
    """The frozen matrices, and what lies where in a replica's row of parameters."""

    def __init__(self, vocab=64, dim=128, rank=16, dtype=torch.bfloat16, seed=0, device="cuda:0"):
        gen = torch.Generator().manual_seed(seed)
        self.vocab, self.dim, self.rank, self.dtype, self.device = vocab, dim, rank, dtype, torch.device(device)

        def matrix(rows, cols, std):
            return (torch.randn(rows, cols, generator=gen) * std).to(self.device, dtype)
        self.E = matrix(vocab, dim, 1.0)
        self.W = {"f": matrix(dim, dim, dim ** -0.5), "x": matrix(dim, dim, dim ** -0.5), "z": matrix(vocab, dim, dim ** -0.5)}
        self.scale = 1.0
        self.place, at = {}, 0
        for name, W in self.W.items():
            for part, shape in (("A", (rank, W.shape[1])), ("B", (W.shape[0], rank))):
                self.place[name + part] = (at, shape)
                at += shape[0] * shape[1]
        self.d, self.stride = at, (at + 63) // 64 * 64

    def start(self, seed=1):
        """One row of parameters: A small and random, B zero, so that the adapted model begins as the frozen one."""
        gen = torch.Generator().manual_seed(seed)
        row = torch.zeros(self.stride)
        for name, (at, shape) in self.place.items():
            if name.endswith("A"):
                row[at:at + shape[0] * shape[1]] = torch.randn(shape[0] * shape[1], generator=gen) * shape[1] ** -0.5
        return row.to(self.device)

    def part(self, rows, name):
        """[K, ...] of the part `name`, inside the rows [K, stride]."""
        at, (n, m) = self.place[name]
        return rows.as_strided((rows.shape[0], n, m), (rows.stride(0), m, 1), rows.storage_offset() + at)

    def segments(self, K, rows):
        return (torch.arange(K + 1, dtype=torch.int32, device=self.device) * rows,
                torch.arange(K, dtype=torch.int32, device=self.device))

    def adapted(self, name, inp, rows, seg):
        return ops.adapter(inp, self.W[name], self.part(rows, name + "A"), self.part(rows, name + "B"), *seg, self.scale)

    def gradient(self, rows, tokens, grads, p, seed, step):
        """Mean loss [K] of the replicas' next tokens, tokens: [K, seqs, length + 1]; d loss / d parameters into `grads`.  The
        dropout mask belongs to `step`: both passes of a sharpness-aware step see the same one."""
        K, seqs, length = tokens.shape[0], tokens.shape[1], tokens.shape[2] - 1
        n = seqs * length
        seg = self.segments(K, n)
        e = self.E[tokens[:, :, :-1].reshape(-1).long()]
        target = tokens[:, :, 1:].reshape(-1).contiguous()
        shape = (K * seqs, length, self.dim)

        f, u_f = self.adapted("f", e, rows, seg)
        x, u_x = self.adapted("x", e, rows, seg)
        h, _, states = ops.recurrence(f.view(shape), x.view(shape), save=True)
        r = ops.dropout(h.view(K, n, self.dim), p, seed, step, residual=e.view(K, n, self.dim)).view(K * n, self.dim)
        z, u_z = self.adapted("z", r, rows, seg)
        out = ops.logprobs(z, target)

        g_logp = torch.full((K * n,), -1.0 / n, device=self.device)
        dz = ops.logprobs_backward(z, target, out.lse, out.entropy, g_logp, out=z)
        dr = self.back("z", r, rows, grads, seg, u_z, dz, True)
        dh = ops.dropout(dr.view(K, n, self.dim), p, seed, step).view(shape)
        df, dx, _ = ops.recurrence_backward(f.view(shape), x.view(shape), dh, states)
        self.back("f", e, rows, grads, seg, u_f, df.view(K * n, self.dim), False)
        self.back("x", e, rows, grads, seg, u_x, dx.view(K * n, self.dim), False)
        return -out.logp.view(K, n).mean(dim=1)

    def back(self, name, inp, rows, grads, seg, u, dy, want_dx):
        dx, _, _ = ops.adapter_backward(inp, self.W[name], self.part(rows, name + "A"), self.part(rows, name + "B"), u, dy, *seg,
                                        self.scale, dA=self.part(grads, name + "A"), dB=self.part(grads, name + "B"), want_dx=want_dx)
        return dx

    def generate(self, row, first, count, top=4, seed=0):
        """`count` tokens after `first` [seqs], each drawn from the `top` most likely; returns them [seqs, count] and the mean
        entropy of the model's choices."""
        seqs = first.shape[0]
        rows, seg = row.view(1, -1), self.segments(1, seqs)
        gen = torch.Generator(device=self.device).manual_seed(seed)
        token, state, made, entropy = first, None, [], 0.0
        for _ in range(count):
            e = self.E[token.long()]
            f, _ = self.adapted("f", e, rows, seg)
            x, _ = self.adapted("x", e, rows, seg)
            h, state, _ = ops.recurrence(f.view(seqs, 1, self.dim), x.view(seqs, 1, self.dim), h0=state)
            z, _ = self.adapted("z", e + h.view(seqs, self.dim), rows, seg)
            best = ops.logprobs(z, top=top)
            pick = torch.multinomial(best.top_logp.exp(), 1, generator=gen)
            token = best.top_ids.gather(1, pick).view(-1)
            made.append(token)
            entropy += float(best.entropy.mean()) / count
        return torch.stack(made, dim=1), entropy


def sequences(K, seqs, length, vocab, step, device):
    """Each token is the one before it plus 1 or 3, in turn: what comes next depends on more than the last token."""
    gen = torch.Generator().manual_seed(1000 + step)
    first = torch.randint(0, vocab, (K, seqs, 1), generator=gen)
    odd = torch.randint(0, 2, (K, seqs, 1), generator=gen)
    t = torch.arange(length + 1)
    return ((first + 2 * t + (t + odd) % 2) % vocab).to(device, torch.int32)


def train(model, K=4, seqs=8, length=64, steps=60, rho=0.05, lr=0.5, momentum=0.9, lam=0.02, period=10, p=0.1, seed=7, say=None):
    """`steps` sharpness-aware steps of K replicas, pulled towards a center that takes their averaged iterates every `period` steps.
    Returns the losses [steps, K] and the center's row of parameters."""
    y = model.start()
    x = y.repeat(K, 1)
    v, S, xt, g1, g2 = (torch.zeros_like(x) for _ in range(5))
    losses = []
    for step in range(steps):
        tokens = sequences(K, seqs, length, model.vocab, step, model.device)
        losses.append(model.gradient(x, tokens, g1, p, seed, step))
        torch.addcdiv(x, g1, g1.norm(dim=1, keepdim=True) + 1e-12, value=rho, out=xt)
        model.gradient(xt, tokens, g2, p, seed, step)
        lsam.lsam_step_grads_static(x, v, S, y, g1, g2, xt, None, [lam] * K, rho, 1e-12, lr, momentum, 1, d=model.d)
        if (step + 1) % period == 0:
            y.copy_(S.sum(dim=0) / (K * period))
            S.zero_()
        if say and (step % 10 == 0 or step == steps - 1):
            say("step %d: loss %s" % (step, " ".join("%.3f" % float(a) for a in losses[-1])))
    return torch.stack(losses), y


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--replicas", type=int, default=4)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--dtype", choices=["bf16", "fp32"], default="bf16")
    args = ap.parse_args()
    model = Model(dtype=torch.bfloat16 if args.dtype == "bf16" else torch.float32)
    print("%d replicas of %d adapter parameters; ln(vocab) = %.3f" % (args.replicas, model.d, math.log(model.vocab)))
    _, y = train(model, K=args.replicas, steps=args.steps, say=print)
    made, entropy = model.generate(y, torch.tensor([0, 17], dtype=torch.int32, device=model.device), 12)
    for row in made.tolist():
        print("generated:", row)
    print("mean entropy %.3f" % entropy)


if __name__ == "__main__":
    main()
