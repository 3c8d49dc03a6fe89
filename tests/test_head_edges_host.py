"""The operators for a head, CPU only: refusals and sizes beside those of test_head_host.py."""
import pytest
import torch


@pytest.mark.parametrize("kind", ["relu", "", None])
def test_unknown_gates_are_refused(kind):
    from paper_2305_11624_amd.gated import Gated, NormGatedBlock
    with pytest.raises(ValueError, match="kind"):
        Gated(4, 24, 8, torch.float32, kind=kind, device="cpu")
    with pytest.raises(ValueError, match="kind"):
        NormGatedBlock(4, 1, 24, 8, dtype=torch.float32, kind=kind, device="cpu")
