"""The operators record nothing for autograd: where torch would, a call is refused instead of cutting the graph without a word."""
import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def calls():
    n = lambda *s: torch.randn(*s, device=DEV)  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)  # noqa: E731
    x, W, A, B, dy = n(6, 8), n(10, 8), n(2, 3, 8), n(2, 10, 3), n(6, 10)
    f, v, dh, h0 = n(2, 4, 5), n(2, 4, 5), n(2, 4, 5), n(2, 5)
    z, tok, g = n(6, 9), i(0, 1, 2, 3, 4, 5), n(6)
    states = ops.recurrence(f, v, h0=h0, save=True).states
    r = ops.logprobs(z, tok)
    seg = dict(seg_begin=i(0, 2, 6), seg_adapter=i(0, 1), scale=1.0)
    u = ops.adapter(x, W, A, B, **seg)[1]
    return [(ops.dropout, dict(x=x, residual=n(6, 8), out=torch.empty_like(x)), dict(p=0.5, seed=1, step=2)),
            (ops.logprobs, dict(logits=z), dict(tokens=tok)),
            (ops.logprobs_backward, dict(logits=z, g_logp=g, g_entropy=n(6), out=torch.empty_like(z)), dict(tokens=tok, lse=r.lse, entropy=r.entropy)),
            (ops.recurrence, dict(f=f, x=v, h0=h0, out=torch.empty_like(f)), dict()),
            (ops.recurrence_backward, dict(f=f, x=v, dh=dh, h0=h0, dlast=n(2, 5), df=torch.empty_like(f), dx=torch.empty_like(f)), dict(states=states)),
            (ops.adapter, dict(x=x, W=W, A=A, B=B, bias=n(10), out=torch.empty_like(dy)), seg),
            (ops.adapter_backward, dict(x=x, W=W, A=A, B=B, dy=dy, dx=torch.empty_like(x), dA=torch.empty_like(A), dB=torch.empty_like(B)),
             dict(seg, u=u))]


def test_tensors_that_want_a_gradient_are_refused_while_gradients_are_recorded():
    for op, tensors, rest in calls():
        op(**tensors, **rest)
        for name, t in tensors.items():
            kw = dict(tensors, **{name: t.detach().requires_grad_()})
            with pytest.raises(lsam.LsamError) as e:
                op(**kw, **rest)
            assert e.value.code == lsam.EINVAL and "gradient" in str(e.value), (op.__name__, name)
            with torch.no_grad():
                op(**kw, **rest)
            with torch.inference_mode():
                op(**dict(kw, **{name: t.detach()}), **rest)
