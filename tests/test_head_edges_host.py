"""The operators for a head, CPU only: refusals and sizes beside those of test_head_host.py."""
import ctypes as C

import pytest
import torch

from paper_2305_11624_amd import binding as B


@pytest.mark.parametrize("kind", ["relu", "", None])
def test_unknown_gates_are_refused(kind):
    from paper_2305_11624_amd.gated import Gated, NormGatedBlock
    with pytest.raises(ValueError, match="kind"):
        Gated(4, 24, 8, torch.float32, kind=kind, device="cpu")
    with pytest.raises(ValueError, match="kind"):
        NormGatedBlock(4, 1, 24, 8, dtype=torch.float32, kind=kind, device="cpu")


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("M", [1, 16, 17, 500])
def test_outputs_in_the_place_of_rows_that_are_still_read_are_refused(M, dtype):
    """Few rows: every workgroup reads all of x; many: tiles read the rows that others write.  (Addresses that are never dereferenced.)"""
    at = [C.c_void_p(4096 * i) for i in range(1, 10)]
    d = B.make_qdesc(M, 64, 64, dtype)
    L, work = B.lib(), (at[8], 1 << 50, None)
    codes, scales, w, ws, rows = at[1], at[2], at[3], at[4], at[0]
    assert L.convbn_flinear_fwd(C.byref(d), rows, codes, scales, w, ws, None, rows, *work) == B.ERR_UNSUPPORTED and "z is x" in B.convbn_last_error()
    assert L.convbn_flinear_bwd(C.byref(d), codes, scales, w, ws, rows, rows, None, None, *work) == B.ERR_UNSUPPORTED and "dx is dz" in B.convbn_last_error()
    assert L.convbn_glu_fwd(C.byref(d), rows, w, None, rows, None, *work) == B.ERR_UNSUPPORTED and "y is x" in B.convbn_last_error()
    assert L.convbn_glu_bwd(C.byref(d), rows, w, None, None, at[5], rows, None, None, *work) == B.ERR_UNSUPPORTED and "dx is x" in B.convbn_last_error()
    n = B.make_norm_desc(M, 4, 64, 8, dtype)
    assert L.convbn_norm_fwd(C.byref(n), rows, None, None, rows, None, *work) == B.ERR_UNSUPPORTED and "y is x" in B.convbn_last_error()


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
def test_no_rows_may_lie_anywhere(dtype):
    d, L = B.make_qdesc(0, 64, 64, dtype), B.lib()
    assert L.convbn_flinear_fwd(C.byref(d), None, None, None, C.c_void_p(4096), C.c_void_p(4096), None, None, None, 0, None) == B.OK
    assert L.convbn_glu_fwd(C.byref(d), None, C.c_void_p(4096), None, None, None, None, 0, None) == B.OK


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,K,N", [(1, 64, 40), (100, 64, 40), (8192, 64, 128), (300, 72, 29)])
def test_a_kept_h_has_no_second_place_in_the_workspace(M, K, N, dtype):
    from paper_2305_11624_amd import gated as G
    h = -(-M * 2 * N * 4 // 256) * 256
    full, less = G.workspace_bytes(M, K, N, dtype), G.workspace_bytes(M, K, N, dtype, keep=True)
    assert full - less == h
    assert G.Gated(M, K, N, dtype, device="cpu").ws.nbytes == less and G.Gated(M, K, N, dtype, device="cpu", keep=False).ws.nbytes == full
    assert G.workspace_bytes(M, K, N, dtype, train=False) == G.workspace_bytes(M, K, N, dtype, train=False, keep=True)
    d = B.make_qdesc(M, K, N, {torch.bfloat16: B.BF16, torch.float32: B.F32}[dtype], act=B.ACT_H_KEPT)
    at = [C.c_void_p(4096 * i) for i in range(1, 9)]
    call = lambda h, work, n: B.lib().convbn_glu_bwd(C.byref(d), at[0], at[1], None, h, at[3], at[4], at[5], None, work, n, None)
    assert call(None, at[7], full) == B.ERR_NULL and "'h'" in B.convbn_last_error()
    assert call(at[2], at[7], less - 1) == B.ERR_WORKSPACE
    for f in (B.lib().convbn_flinear_fwd, B.lib().convbn_qlinear_fwd):      # (the bit is the gated product's)
        assert f(C.byref(d), *[at[0]] * 7, at[7], full, None) == B.ERR_UNSUPPORTED


def test_blocks_that_keep_h_have_the_smaller_workspace():
    from paper_2305_11624_amd.gated import NormGatedBlock
    sizes = (4, 25, 64, 256)
    kept, again = (NormGatedBlock(*sizes, keep=k, device="cpu") for k in (True, False))
    assert again.gated.ws.nbytes - kept.gated.ws.nbytes > 0
    NormGatedBlock(*sizes, keep=True, device="cpu", share=again)
    with pytest.raises(ValueError, match="ws"):
        NormGatedBlock(*sizes, keep=False, device="cpu", share=kept)
