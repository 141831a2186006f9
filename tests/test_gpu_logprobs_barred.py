"""lsam_logprobs where a row's own token is barred: its log probability is -inf, and the gradient is the formula's with p = 0 there --
the token's own logit receives g_logp, other barred ones nothing.  Bounds as the finite rows' tests derive them."""
import math

import pytest
import torch

from paper_2509_03110_amd import ops
from test_gpu_logprobs import B16, DEV, F32, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, B16])
@pytest.mark.parametrize("rows,V", [(4, 10), (6, 5000), (3, 40001)])
def test_a_barred_token_of_its_own(dtype, rows, V):
    z, tokens, gl, ge = make(rows, V, dtype, seed=V)
    z, tokens = z.clone(), torch.arange(rows, device=DEV, dtype=torch.int32) * 2
    z[:, 1] = -math.inf
    at = tokens.long()[:, None]
    z.scatter_(1, at, -math.inf)
    r = check(z, tokens, 3, gl, ge)
    dz = ops.logprobs_backward(z, tokens, r.lse, r.entropy, gl, ge)
    assert bool((r.logp == -math.inf).all())
    assert torch.equal(dz.gather(1, at)[:, 0], gl.to(dtype)) and bool((dz[:, 1] == 0).all())
