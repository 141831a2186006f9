"""Heads of no numbers are refused as other widths outside of the range are."""
import pytest
import torch

from paper_2509_03110_amd import lsam, ops

pytestmark = pytest.mark.gpu


def test_heads_of_no_numbers():
    e = torch.empty(4, 2, 0, device="cuda:0")
    off = torch.tensor([0, 4], device="cuda:0")
    lse = torch.zeros(2, 4, device="cuda:0")
    n = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    for call in (lambda: ops.attention(e, e, e, off), lambda: ops.attention_backward(e, e, e, off, e, lse, e),
                 lambda: ops.attention_step(e, e[:, None], e[:, None], n)):
        with pytest.raises(lsam.LsamError) as r:
            call()
        assert r.value.code == lsam.EINVAL and "dim" in str(r.value)
