"""Edges of the operators for a head on the GPU: every byte of kept 8-bit floating-point rows."""
import pytest
import torch

import head_ref as R
from head_ref import DT

pytestmark = pytest.mark.gpu


# ---- rows in 8-bit floating point -----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 5, 16, 40])
@pytest.mark.parametrize("K", [1, 64, 130, 136, 300, 512, 513, 600])
def test_rows_that_forward_keeps_are_those_of_pack(K, M, dtype):
    """Codes and scales byte by byte, what lies past the last channel and the last block among them, however many rows there are."""
    from paper_2305_11624_amd import quant as Q
    x = torch.randn(M, K, generator=R.gen(K + M)).to("cuda", DT[dtype])
    lay = Q.F8Linear(M, K, 8, DT[dtype])
    lay.pack_weight(torch.ones(8, K, device="cuda", dtype=DT[dtype]))
    lay.codes.fill_(77)
    lay.scales.fill_(3)
    lay.forward(x)
    ck = Q.F8Checkpoint(M, K, DT[dtype])
    ck.codes.fill_(99)
    ck.scales.fill_(5)
    ck.pack(x)
    assert torch.equal(lay.codes, ck.codes) and torch.equal(lay.scales, ck.scales)
    assert (lay.scales[:, -(-K // 128):] == 127).all()
