"""The operators for a head, CPU only: sizes, and every refusal before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2305_11624_amd import binding as B

import head_ref as R

OKP = C.c_void_p(4096)      # never dereferenced: validation fails first
ODD, HALF = C.c_void_p(4097), C.c_void_p(4104)
NEED = 1 << 50


def _qdesc(**change):
    return B.make_qdesc(**dict(dict(M=8, K=64, N=32, dtype=B.BF16), **change))


def _ndesc(**change):
    return B.make_norm_desc(**dict(dict(M=2, P=9, channels=64, groups=8, dtype=B.BF16), **change))


def _call(name, tensors, ws):
    """A call with every pointer in place; keywords by position replace some."""
    def f(d, work=OKP, nbytes=NEED, **change):
        p = [OKP] * tensors
        for k, v in change.items():
            p[int(k[1:])] = v
        return getattr(B.lib(), name)(C.byref(d) if d is not None else None, *p, *((work, nbytes) if ws else ()), None)
    return f


fpack, funpack = _call("convbn_fpack", 3, False), _call("convbn_funpack", 3, False)
ffwd, fbwd = _call("convbn_flinear_fwd", 7, True), _call("convbn_flinear_bwd", 8, True)
gfwd, gbwd = _call("convbn_glu_fwd", 5, True), _call("convbn_glu_bwd", 8, True)
nfwd, nbwd = _call("convbn_norm_fwd", 5, True), _call("convbn_norm_bwd", 8, True)


def test_scale_bytes_are_whole_words():
    assert [B.convbn_fscale_bytes(k) for k in (-1, 0, 1, 128, 129, 512, 513, 4096)] == [0, 0, 4, 4, 4, 4, 8, 32]


def test_descriptor_mirror_has_the_size_of_the_struct():
    assert C.sizeof(B.NormDesc) == 72 and C.sizeof(B.NormDesc) not in (C.sizeof(B.QDesc), C.sizeof(B.Desc))


def test_the_definition_of_the_codes():
    """The plain packing against what PyTorch's own type stands for."""
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(v, R.e4m3_values(), equal_nan=True)
    x = np.random.default_rng(0).standard_normal((4, 300)).astype(np.float32)
    q, s = R.f8_pack(x)
    y = R.f8_values(q, s)
    assert np.abs(y - x).max() <= 2.0 ** -4 * np.abs(x).max() and (s >= 11).all()
    assert np.array_equal(R.f8_pack(y.astype(np.float32))[0], q)      # what is held stays as it is


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), B.ERR_SHAPE), (dict(K=0), B.ERR_SHAPE), (dict(N=0), B.ERR_SHAPE), (dict(dtype=2), B.ERR_UNSUPPORTED),
    (dict(ldx=63), B.ERR_SHAPE), (dict(ldz=31), B.ERR_SHAPE), (dict(ldx=-64), B.ERR_SHAPE), (dict(act=1), B.ERR_UNSUPPORTED),
    (dict(act=16), B.ERR_UNSUPPORTED), (dict(act=8), B.ERR_NULL), (dict(K=131073), B.ERR_UNSUPPORTED),
    (dict(N=(1 << 20) + 1), B.ERR_UNSUPPORTED), (dict(M=(1 << 30) + 1), B.ERR_UNSUPPORTED), (dict(ldx=1 << 41), B.ERR_UNSUPPORTED),
    (dict(M=1 << 30, K=257), B.ERR_UNSUPPORTED), (dict(M=1 << 30, N=257), B.ERR_UNSUPPORTED)])
def test_bad_descriptors_of_the_products(change, code):
    d = _qdesc(**change)
    assert ffwd(d) == code and fbwd(d) == code and gfwd(d) == code and gbwd(d) == code
    for f in (B.convbn_flinear_workspace_bytes, B.convbn_glu_workspace_bytes):
        assert f(d, B.PASS_FWD) == 0 == f(d, B.PASS_BWD)
    assert len(B.convbn_last_error()) > 4


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), B.ERR_SHAPE), (dict(P=0), B.ERR_SHAPE), (dict(channels=0), B.ERR_SHAPE), (dict(groups=0), B.ERR_SHAPE), (dict(groups=7), B.ERR_SHAPE),
    (dict(dtype=2), B.ERR_UNSUPPORTED), (dict(f=4), B.ERR_UNSUPPORTED), (dict(f=-1), B.ERR_UNSUPPORTED), (dict(eps=0.0), B.ERR_SHAPE), (dict(eps=-1.0), B.ERR_SHAPE),
    (dict(eps=float("nan")), B.ERR_SHAPE), (dict(eps=float("inf")), B.ERR_SHAPE), (dict(act=4), B.ERR_UNSUPPORTED), (dict(act=8), B.ERR_NULL),
    (dict(ldx=63), B.ERR_SHAPE), (dict(ldy=63), B.ERR_SHAPE), (dict(ldx=-64), B.ERR_SHAPE), (dict(ldx=1 << 33), B.ERR_UNSUPPORTED),
    (dict(channels=(1 << 20) + 8), B.ERR_UNSUPPORTED), (dict(M=1 << 20, P=1 << 11), B.ERR_UNSUPPORTED), (dict(M=1 << 31), B.ERR_UNSUPPORTED),
    (dict(M=1 << 28), B.ERR_UNSUPPORTED), (dict(M=1 << 62, P=1 << 62), B.ERR_UNSUPPORTED), (dict(M=1 << 22, P=1 << 8, channels=512), B.ERR_UNSUPPORTED)])
def test_bad_descriptors_of_group_norm(change, code):
    d = _ndesc(**change)
    assert nfwd(d) == code and nbwd(d) == code
    assert B.convbn_norm_workspace_bytes(d, B.PASS_FWD) == 0 == B.convbn_norm_workspace_bytes(d, B.PASS_BWD)


def test_reserved_fields_missing_descriptors_unknown_gates():
    d = _qdesc()
    d.reserved = 1
    assert ffwd(d) == gfwd(d) == fpack(d) == B.ERR_UNSUPPORTED
    n = _ndesc()
    n.reserved = 1
    assert nfwd(n) == B.ERR_UNSUPPORTED
    for f in (fpack, funpack, ffwd, fbwd, gfwd, gbwd, nfwd, nbwd):
        assert f(None) == B.ERR_NULL
    assert gfwd(_qdesc(gate=2)) == B.ERR_UNSUPPORTED == gbwd(_qdesc(gate=2))
    d = _qdesc(act=B.ACT_ADD_OUT)
    d.add_out = 4096
    assert gfwd(d) == B.ERR_UNSUPPORTED


def test_missing_and_misaligned_pointers():
    d, n = _qdesc(), _ndesc()
    for f in (fpack, funpack):
        for i in range(3):
            assert f(d, **{"p%d" % i: None}) == B.ERR_NULL
    assert fpack(d, p0=ODD) == fpack(d, p1=HALF) == fpack(d, p2=C.c_void_p(4098)) == B.ERR_UNSUPPORTED
    assert ffwd(d, p0=None, p1=None, p2=None) == B.ERR_NULL and ffwd(d, p2=None) == B.ERR_NULL and "together" in B.convbn_last_error()
    assert ffwd(d, p3=None) == ffwd(d, p4=None) == ffwd(d, p6=None) == B.ERR_NULL
    assert ffwd(d, p1=HALF) == ffwd(d, p3=HALF) == ffwd(d, p0=ODD) == ffwd(d, p6=ODD) == B.ERR_UNSUPPORTED
    assert fbwd(d, p4=None) == fbwd(d, p5=None, p6=None, p7=None) == fbwd(d, p0=None) == fbwd(d, p2=None) == B.ERR_NULL
    assert fbwd(d, p4=HALF) == B.ERR_UNSUPPORTED and "16-byte" in B.convbn_last_error()      # read in place: N, ldz multiples of 8
    assert gfwd(d, p0=None) == gfwd(d, p1=None) == gfwd(d, p3=None) == B.ERR_NULL
    assert gfwd(d, p0=HALF) == gfwd(d, p1=HALF) == gfwd(d, p3=ODD) == gfwd(d, p4=ODD) == gfwd(d, p2=ODD) == B.ERR_UNSUPPORTED
    assert gbwd(d, p0=None) == gbwd(d, p1=None) == gbwd(d, p4=None) == gbwd(d, p5=None, p6=None, p7=None) == B.ERR_NULL
    assert gbwd(d, p0=HALF) == gbwd(d, p1=HALF) == gbwd(d, p3=ODD) == gbwd(d, p4=ODD) == B.ERR_UNSUPPORTED
    f = _qdesc(dtype=B.F32)
    assert gfwd(f, p0=C.c_void_p(4098)) == gbwd(f, p5=C.c_void_p(4098)) == B.ERR_UNSUPPORTED
    assert nfwd(n, p0=None) == nfwd(n, p3=None) == B.ERR_NULL and nfwd(n, p0=ODD) == nfwd(n, p1=ODD) == nfwd(n, p4=ODD) == B.ERR_UNSUPPORTED
    assert nbwd(n, p0=None) == nbwd(n, p3=None) == nbwd(n, p4=None) == nbwd(n, p5=None, p6=None, p7=None) == B.ERR_NULL
    assert nbwd(n, p4=ODD) == nbwd(n, p5=ODD) == nbwd(n, p6=C.c_void_p(4098)) == B.ERR_UNSUPPORTED


def test_workspace_is_asked_for_and_checked():
    for f, need, d in ((ffwd, B.convbn_flinear_workspace_bytes(_qdesc(M=100), B.PASS_FWD), _qdesc(M=100)),
                       (gbwd, B.convbn_glu_workspace_bytes(_qdesc(M=100), B.PASS_BWD), _qdesc(M=100)),
                       (nbwd, B.convbn_norm_workspace_bytes(_ndesc(), B.PASS_BWD), _ndesc())):
        none = dict(p1=None, p2=None) if f is ffwd else {}
        assert need > 0 and need % 256 == 0
        assert f(d, work=None, nbytes=0, **none) == B.ERR_WORKSPACE
        assert f(d, nbytes=need - 1, **none) == B.ERR_WORKSPACE
        assert f(d, work=HALF, **none) == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("M,K,N", [(0, 64, 40), (1, 1, 1), (0, 1, 1), (1 << 30, 16, 1), (1 << 30, 256, 256), (1, 131072, 1 << 20), (4097, 4096, 4096)])
def test_workspace_query_of_any_size(M, K, N, dtype):
    d = _qdesc(M=M, K=K, N=N, dtype=dtype)
    for p in (B.PASS_FWD, B.PASS_BWD):
        assert B.convbn_flinear_workspace_bytes(d, p) % 256 == 0 and B.convbn_glu_workspace_bytes(d, p) % 256 == 0


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("M,P,Ch,G", [(0, 1, 1, 1), (1, 1, 1 << 20, 1 << 20), (1 << 30, 1, 256, 1), (1 << 10, 1 << 20, 256, 256), (1, 1 << 30, 256, 1)])
def test_norm_workspace_query_of_any_size(M, P, Ch, G, dtype):
    d = _ndesc(M=M, P=P, channels=Ch, groups=G, dtype=dtype)
    for p in (B.PASS_FWD, B.PASS_BWD):
        assert B.convbn_norm_workspace_bytes(d, p) % 256 == 0


def test_tensors_that_do_not_fit_are_refused_by_the_classes():
    from paper_2305_11624_amd import gated, norm, quant as Q
    lin = Q.F8Linear(4, 300, 8, torch.float32, device="cpu")
    with pytest.raises(RuntimeError):
        lin.forward(torch.zeros(4, 300))
    with pytest.raises(ValueError):
        lin.set_weight(torch.zeros(8, 304, dtype=torch.uint8), torch.zeros(8, dtype=torch.float32))      # the other form's scales
    w = Q.new_f8_codes(8, 300, "cpu")
    assert w[0].shape == (8, 304) and w[1].shape == (8, 4)
    lin.set_weight(*w)
    with pytest.raises(ValueError):
        lin.forward(torch.zeros(4, 299))
    with pytest.raises(ValueError):
        lin.forward(torch.zeros(4, 300), add=torch.zeros(4, 9))
    assert lin.saved_bytes() == 4 * (304 + 4)
    g = gated.Gated(4, 24, 8, torch.float32, device="cpu")
    for x, W, b in ((torch.zeros(4, 23), torch.zeros(16, 24), None), (torch.zeros(4, 24), torch.zeros(8, 24), None),
                    (torch.zeros(4, 24), torch.zeros(16, 24), torch.zeros(8)), (torch.zeros(4, 24, dtype=torch.bfloat16), torch.zeros(16, 24), None),
                    (None, torch.zeros(16, 24), None), (torch.zeros(4, 24), torch.zeros(16, 48)[:, ::2], None)):
        with pytest.raises(ValueError):
            g.forward(x, W, b)
    with pytest.raises(ValueError):
        g.backward(torch.zeros(4, 24), torch.zeros(16, 24), torch.zeros(4, 8), add=torch.zeros(4, 23))
    with pytest.raises(RuntimeError):
        gated.Gated(4, 24, 8, torch.float32, train=False, device="cpu").backward(torch.zeros(4, 24), torch.zeros(16, 24), torch.zeros(4, 8))
    assert g.saved_bytes() == 4 * 16 * 4 and gated.Gated(4, 24, 8, torch.float32, keep=False, device="cpu").saved_bytes() == 0
    n = norm.GroupNorm(2, 9, 24, 3, torch.float32, device="cpu")
    for x, ga in ((torch.zeros(18, 23), None), (torch.zeros(17, 24), None), (torch.zeros(18, 24), torch.zeros(23)), (torch.zeros(18, 24).double(), None), (None, None)):
        with pytest.raises(ValueError):
            n.forward(x, ga)
    with pytest.raises(ValueError):
        n.backward(torch.zeros(18, 24), None, None, torch.zeros(18, 24), add=torch.zeros(18, 25))
    with pytest.raises(ValueError):
        norm.GroupNorm(2, 9, 24, 3, torch.float32, act="tanh", device="cpu")
    with pytest.raises(RuntimeError):
        norm.GroupNorm(2, 9, 24, 3, torch.float32, train=False, device="cpu").backward(torch.zeros(18, 24), None, None, torch.zeros(18, 24))
    with pytest.raises(TypeError):
        norm.GroupNorm(2, 9, 24, 3, torch.float16, device="cpu")
    for f in (lambda ws: gated.Gated(400, 24, 8, torch.float32, device="cpu", ws=ws), lambda ws: norm.GroupNorm(2, 9, 24, 3, torch.float32, device="cpu", ws=ws)):
        with pytest.raises(ValueError):
            f(torch.empty(16, dtype=torch.uint8))


def test_host_tensors_are_refused():
    from paper_2305_11624_amd import gated, norm
    with pytest.raises(AssertionError):
        gated.Gated(4, 24, 8, torch.float32, train=False, device="cpu").forward(torch.zeros(4, 24), torch.zeros(16, 24))
    with pytest.raises(AssertionError):
        norm.GroupNorm(2, 9, 24, 3, torch.float32, train=False, device="cpu").forward(torch.zeros(18, 24))


def test_native_call_takes_the_norm_descriptor_only():
    B.lib()
    at = B._at.convbn_norm_fwd
    assert B._call_norm(at, _ndesc(), "xvvys", None, None, None, None, None, None, 0) == B.ERR_NULL
    for bad in (None, b"\0" * 8, B.Desc(), _qdesc()):
        with pytest.raises(TypeError):
            B._call_norm(at, bad, "xvvys", None, None, None, None, None, None, 0)
    with pytest.raises(TypeError):
        B._call_rows(at, _ndesc(), "xvvys", None, None, None, None, None, None, 0)


def test_group_norm_in_place_is_refused():
    """Large parts take two launches, the second of which reads every group's first value again."""
    assert nfwd(_ndesc()) == nfwd(_ndesc(M=1, P=5000, groups=1)) == B.ERR_UNSUPPORTED and "y is x" in B.convbn_last_error()
    assert nfwd(_ndesc(M=0), p0=None, p3=None) == B.OK
