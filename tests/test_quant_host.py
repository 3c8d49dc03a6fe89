"""The 8-bit rows, CPU only: sizes, and every refusal before anything is launched."""
import ctypes as C

import pytest
import torch

from paper_2305_11624_amd import binding as B

OKP = C.c_void_p(4096)      # never dereferenced: validation fails first
NEED = 1 << 40


def _qdesc(**change):
    kw = dict(M=8, K=64, N=32, dtype=B.BF16)
    kw.update(change)
    return B.make_qdesc(**kw)


def _fwd(d, x=OKP, codes=OKP, scales=OKP, w=OKP, ws=OKP, b=None, z=OKP, work=OKP, nbytes=NEED):
    return B.lib().convbn_qlinear_fwd(C.byref(d), x, codes, scales, w, ws, b, z, work, nbytes, None)


def _bwd(d, codes=OKP, scales=OKP, w=OKP, ws=OKP, dz=OKP, dx=OKP, dW=OKP, db=OKP, work=OKP, nbytes=NEED):
    return B.lib().convbn_qlinear_bwd(C.byref(d), codes, scales, w, ws, dz, dx, dW, db, work, nbytes, None)


def _gate(d, h=OKP, hc=OKP, hs=OKP, y=OKP, yc=OKP, ys=OKP):
    return B.lib().convbn_qgate_fwd(C.byref(d), h, hc, hs, y, yc, ys, None)


def test_row_bytes_are_whole_16_byte_pieces():
    assert [B.convbn_qrow_bytes(k) for k in (-1, 0, 1, 15, 16, 17, 72, 4096)] == [0, 0, 16, 16, 16, 32, 80, 4096]


def test_descriptor_mirror_has_the_size_of_the_struct():
    assert C.sizeof(B.QDesc) == 64 and C.sizeof(B.Desc) != C.sizeof(B.QDesc)


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), B.ERR_SHAPE), (dict(K=0), B.ERR_SHAPE), (dict(N=0), B.ERR_SHAPE), (dict(dtype=2), B.ERR_UNSUPPORTED),
    (dict(ldx=63), B.ERR_SHAPE), (dict(ldz=31), B.ERR_SHAPE), (dict(ldx=-64), B.ERR_SHAPE), (dict(act=1), B.ERR_UNSUPPORTED),
    (dict(act=16), B.ERR_UNSUPPORTED), (dict(act=4), B.ERR_NULL), (dict(act=8), B.ERR_NULL), (dict(K=131073), B.ERR_UNSUPPORTED), (dict(N=(1 << 20) + 1), B.ERR_UNSUPPORTED),
    (dict(M=(1 << 30) + 1), B.ERR_UNSUPPORTED), (dict(ldx=1 << 41), B.ERR_UNSUPPORTED), (dict(M=1 << 30, K=257), B.ERR_UNSUPPORTED),
    (dict(M=1 << 30, N=257), B.ERR_UNSUPPORTED)])
def test_bad_descriptors_of_a_linear_block(change, code):
    d = _qdesc(**change)
    assert _fwd(d) == code and _bwd(d) == code
    assert B.convbn_qlinear_workspace_bytes(d, B.PASS_FWD) == 0 == B.convbn_qlinear_workspace_bytes(d, B.PASS_BWD)
    assert len(B.convbn_last_error()) > 4


def test_reserved_field_and_missing_descriptor():
    d = _qdesc()
    d.reserved = 1
    assert _fwd(d) == B.ERR_UNSUPPORTED and _gate(d) == B.ERR_UNSUPPORTED
    L = B.lib()
    assert L.convbn_qpack(None, OKP, OKP, OKP, None) == B.ERR_NULL
    assert L.convbn_qunpack(None, OKP, OKP, OKP, None) == B.ERR_NULL
    assert L.convbn_qlinear_fwd(None, OKP, OKP, OKP, OKP, OKP, None, OKP, OKP, NEED, None) == B.ERR_NULL
    assert L.convbn_qlinear_bwd(None, OKP, OKP, OKP, OKP, OKP, OKP, OKP, OKP, OKP, NEED, None) == B.ERR_NULL
    assert L.convbn_qgate_fwd(None, OKP, None, None, OKP, None, None, None) == B.ERR_NULL
    assert L.convbn_qgate_bwd(None, OKP, OKP, OKP, OKP, None) == B.ERR_NULL


def test_missing_and_misaligned_pointers():
    d = _qdesc()
    assert _fwd(d, x=None, codes=None, scales=None) == B.ERR_NULL      # neither rows nor codes
    assert _fwd(d, scales=None) == B.ERR_NULL and "together" in B.convbn_last_error()
    assert _fwd(d, w=None) == B.ERR_NULL and _fwd(d, ws=None) == B.ERR_NULL and _fwd(d, z=None) == B.ERR_NULL
    assert _fwd(d, codes=C.c_void_p(4104)) == B.ERR_UNSUPPORTED and _fwd(d, w=C.c_void_p(4104)) == B.ERR_UNSUPPORTED
    assert _fwd(d, x=C.c_void_p(4097)) == B.ERR_UNSUPPORTED and _fwd(d, z=C.c_void_p(4097)) == B.ERR_UNSUPPORTED
    assert _bwd(d, dz=None) == B.ERR_NULL and _bwd(d, dx=None, dW=None, db=None) == B.ERR_NULL
    assert _bwd(d, codes=None) == B.ERR_NULL and _bwd(d, w=None) == B.ERR_NULL
    assert _bwd(_qdesc(dtype=B.F32), dz=C.c_void_p(4098)) == B.ERR_UNSUPPORTED
    assert _bwd(d, dz=C.c_void_p(4104)) == B.ERR_UNSUPPORTED and "16-byte" in B.convbn_last_error()   # read in place: N, ldz multiples of 8
    for name in ("convbn_qpack", "convbn_qunpack"):
        f = getattr(B.lib(), name)
        for i in range(3):
            p = [OKP] * 3
            p[i] = None
            assert f(C.byref(d), *p, None) == B.ERR_NULL
    assert B.lib().convbn_qpack(C.byref(d), C.c_void_p(4097), OKP, OKP, None) == B.ERR_UNSUPPORTED


def test_gate_refusals():
    assert _gate(_qdesc(gate=2)) == B.ERR_UNSUPPORTED
    assert _gate(_qdesc(ldx=127)) == B.ERR_SHAPE and _gate(_qdesc(ldz=63)) == B.ERR_SHAPE
    d = _qdesc()
    assert _gate(d, h=None) == B.ERR_NULL and _gate(d, hs=None) == B.ERR_NULL and _gate(d, ys=None) == B.ERR_NULL
    assert _gate(d, y=None, yc=None, ys=None) == B.ERR_NULL
    assert _gate(d, h=C.c_void_p(4097)) == B.ERR_UNSUPPORTED
    assert B.lib().convbn_qgate_bwd(C.byref(d), OKP, OKP, OKP, None, None) == B.ERR_NULL


def test_workspace_is_asked_for_and_checked():
    d = _qdesc(M=100)      # (few rows are packed by the product itself)
    need = B.convbn_qlinear_workspace_bytes(d, B.PASS_FWD)
    assert need >= 100 * 64 + 100 * 4
    assert _fwd(d, codes=None, scales=None, work=None, nbytes=0) == B.ERR_WORKSPACE
    assert _fwd(d, codes=None, scales=None, nbytes=need - 1) == B.ERR_WORKSPACE
    assert _fwd(d, codes=None, scales=None, work=C.c_void_p(4104)) == B.ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", [B.F32, B.BF16])
@pytest.mark.parametrize("M,K,N", [(0, 64, 40), (1, 1, 1), (0, 1, 1), (1 << 30, 16, 1), (1 << 30, 256, 256), (1, 131072, 1 << 20), (4097, 4096, 4096)])
def test_workspace_query_of_any_size(M, K, N, dtype):
    d = _qdesc(M=M, K=K, N=N, dtype=dtype)
    for p in (B.PASS_FWD, B.PASS_BWD):
        assert B.convbn_qlinear_workspace_bytes(d, p) % 256 == 0


def test_gradients_that_are_read_in_place_need_no_copy():
    n = {N: B.convbn_qlinear_workspace_bytes(_qdesc(M=100000, K=64, N=N), B.PASS_BWD) for N in (32, 31)}
    assert n[31] >= n[32] + 100000 * 30 * 2      # (less other scratch, which goes by N)
    assert B.convbn_qlinear_workspace_bytes(_qdesc(M=100000, K=64, N=32, ldz=37), B.PASS_BWD) == n[32] + 100000 * 32 * 2


def test_native_call_takes_the_descriptors_rows_only():
    B.lib()
    call, at = B._call_rows, B._at.convbn_qpack
    assert call(at, _qdesc(), "xcs", None, None, None, B._NO_WS, 0) == B.ERR_NULL
    for bad in (None, b"\0" * 8, B.Desc()):
        with pytest.raises(TypeError):
            call(at, bad, "xcs", None, None, None, B._NO_WS, 0)
    for kinds in ("xc", None):
        with pytest.raises(TypeError):
            call(at, _qdesc(), kinds, None, None, None, B._NO_WS, 0)
    with pytest.raises(TypeError):
        B._call(at, _qdesc(), None, None, None, None, B._NO_WS, 0)
    with pytest.raises(AssertionError):
        call(at, _qdesc(), "xcs", torch.zeros(8, 64, dtype=torch.bfloat16), None, None, B._NO_WS, 0)
    with pytest.raises(TypeError):
        call(at, _qdesc(), "xxxxx", *[None] * 5, B._NO_WS, 0)   # (no entry point takes five)


GOOD = dict(x=(torch.bfloat16, 8, 64), z=(torch.bfloat16, 8, 32), h=(torch.bfloat16, 8, 128), y=(torch.bfloat16, 8, 64),
            W=(torch.bfloat16, 32, 64), c=(torch.int8, 8, 64), d=(torch.uint8, 32, 64), e=(torch.int8, 16, 64))


@pytest.mark.parametrize("kind", sorted(GOOD))
def test_tensors_are_checked_against_the_descriptor(kind):
    """A tensor of the wrong type, size or stride is a ValueError; the right one gets as far as the check for the device."""
    B.lib()
    call, at, d = B._call_rows, B._at.convbn_qpack, _qdesc()
    dt, rows, width = GOOD[kind]
    other = torch.float32 if dt is torch.bfloat16 else torch.int16
    good = torch.zeros(rows, width, dtype=dt)
    for bad in (good[:-1], good[:, :-1], good.to(other), torch.zeros(rows, width + 8, dtype=dt)[:, :width], torch.zeros(width, rows, dtype=dt).t(),
                good.view(1, rows, width), good.view(-1)):
        with pytest.raises(ValueError):
            call(at, d, kind + "cs", bad, None, None, B._NO_WS, 0)
    with pytest.raises(AssertionError):
        call(at, d, kind + "cs", good, None, None, B._NO_WS, 0)
    if kind in "xzhy":      # rows of a wider buffer, where the descriptor says so
        d.ldx, d.ldz = (width + 8, 0) if kind in "xh" else (0, width + 8)
        with pytest.raises(AssertionError):
            call(at, d, kind + "cs", torch.zeros(rows, width + 8, dtype=dt)[:, :width], None, None, B._NO_WS, 0)
        with pytest.raises(ValueError):
            call(at, d, kind + "cs", good, None, None, B._NO_WS, 0)


@pytest.mark.parametrize("kind,n", [("s", 8), ("n", 32), ("t", 16)])
def test_vectors_are_checked_against_the_descriptor(kind, n):
    B.lib()
    call, at, d = B._call_rows, B._at.convbn_qpack, _qdesc()
    for bad in (torch.zeros(n + 1), torch.zeros(n - 1), torch.zeros(n, dtype=torch.float64), torch.zeros(2 * n)[::2]):
        with pytest.raises(ValueError):
            call(at, d, "xc" + kind, None, None, bad, B._NO_WS, 0)
    with pytest.raises(AssertionError):
        call(at, d, "xc" + kind, None, None, torch.zeros(n), B._NO_WS, 0)


def test_objects_check_their_arguments():
    from paper_2305_11624_amd import quant as Q
    with pytest.raises(TypeError):
        Q.Checkpoint(4, 8, torch.float16, device="cpu")
    with pytest.raises(KeyError):
        Q.Gate(4, 8, kind="relu", device="cpu")
    lin = Q.Linear(4, 24, 8, torch.float32, train=False, device="cpu")
    x = torch.zeros(4, 24)
    with pytest.raises(RuntimeError):
        lin.forward(x)                                   # no weight yet
    with pytest.raises(ValueError):
        lin.set_weight(torch.zeros(8, 24, dtype=torch.int8), torch.zeros(8))      # rows are 32 bytes
    lin.set_weight(*Q.new_codes(8, 24, "cpu"))
    for bad in (x[:, :23], x.bfloat16(), torch.zeros(4, 32)[:, :24], x[:3]):
        with pytest.raises(ValueError):
            lin.forward(bad)
    with pytest.raises(ValueError):
        lin.forward(x, b=torch.zeros(7))
    with pytest.raises(RuntimeError):
        lin.backward(torch.zeros(4, 8))
    with pytest.raises(AssertionError):
        lin.forward(x)                                   # right in everything, but on the host


@pytest.mark.parametrize("M", [1, 4])
def test_addends_are_checked_like_every_other_tensor(M):
    """An addend goes to the kernel as an address: its type, size, strides and device are looked at first, for a single row too."""
    from paper_2305_11624_amd import quant as Q
    lin = Q.Linear(M, 24, 8, torch.float32, device="cpu", gap=3)
    lin.set_weight(*Q.new_codes(8, 24, "cpu"))

    def rows(width, gap=3, dtype=torch.float32, device="cpu"):
        return torch.zeros(M, width + gap, dtype=dtype, device=device)[:, :width]

    x, dz = rows(24), rows(8)
    for call, width in ((lambda a: lin.forward(x, add=a), 8), (lambda a: lin.forward_packed(lin.codes, lin.scales, add=a), 8),
                        (lambda a: lin.backward(dz, add=a), 24)):
        bad = [torch.zeros(M, 2 * (width + 3))[:, :2 * width:2],      # every other element of a row
               torch.zeros(1, 1).expand(M, width), rows(width + 1), rows(width).t(), rows(width, dtype=torch.bfloat16),
               rows(width).view(1, M, width), rows(width, device="meta")]
        if M > 1:
            bad.append(rows(width, gap=0))      # (a single row is as far from the next as one likes)
        for a in bad:
            with pytest.raises(ValueError):
                call(a)
    with pytest.raises(AssertionError):
        lin.forward(x, add=rows(8))            # right in everything, but on the host
    if M == 1:
        with pytest.raises(AssertionError):
            lin.forward(x, add=rows(8, gap=0))


def test_no_rows_need_no_addend():
    """M = 0 is no error, whatever the call adds: a tensor without rows has no memory either."""
    d = _qdesc(M=0, act=4)
    assert _fwd(d, x=None, codes=None, scales=None, z=None, work=None, nbytes=0) == B.OK
    assert _fwd(_qdesc(act=4)) == B.ERR_NULL and _bwd(_qdesc(act=8)) == B.ERR_NULL
    for act in (4, 8):      # (as far as the next check)
        assert _bwd(_qdesc(M=0, act=act), dz=None, db=None, dW=None, dx=C.c_void_p(4097)) == B.ERR_UNSUPPORTED
        assert "dx" in B.convbn_last_error()


def test_what_a_layer_packs_into_is_its_own(monkeypatch):
    """By the tensors that the calls get: outputs of packing are never tensors that the caller handed over."""
    from paper_2305_11624_amd import quant as Q
    seen = []
    monkeypatch.setattr(B, "convbn_qlinear_fwd", lambda d, x, codes, scales, *rest: seen.append((x, codes, scales)))
    monkeypatch.setattr(B, "convbn_qlinear_bwd", lambda d, codes, scales, *rest: seen.append((None, codes, scales)))
    lin = Q.Linear(4, 24, 8, torch.float32, device="cpu")
    given, w = Q.new_codes(4, 24, "cpu"), Q.new_codes(8, 24, "cpu")
    lin.set_weight(*w)
    x, dz = torch.zeros(4, 24), torch.zeros(4, 8)
    lin.forward_packed(*given)
    lin.backward(dz)
    assert all(s[1] is given[0] and s[2] is given[1] for s in seen[-2:])
    lin.forward(x)
    assert seen[-1][1] is not given[0] and seen[-1][2] is not given[1]
    own = seen[-1]
    lin.backward(dz)
    assert seen[-1][1] is own[1] and seen[-1][2] is own[2]
    serve = Q.Linear(4, 24, 8, torch.float32, train=False, device="cpu")
    serve.set_weight(*w)
    serve.forward(x)
    serve.forward_packed(*given)
    serve.forward(x)
    assert seen[-1][1] is None and seen[-1][2] is None      # nothing is kept
    never = Q.Linear(4, 24, 8, torch.float32, packed=True, device="cpu")
    never.set_weight(*w)
    assert never.codes is None and never.saved_bytes() == lin.saved_bytes() == 4 * (32 + 4)
    never.forward_packed(*given)
    never.backward(dz)
    assert seen[-1][1] is given[0]
    with pytest.raises(RuntimeError):
        never.forward(x)


def test_a_weight_is_packed_into_the_layers_own_buffers(monkeypatch):
    from paper_2305_11624_amd import quant as Q
    seen = []
    monkeypatch.setattr(B, "convbn_qpack", lambda d, x, codes, scales, stream=None: seen.append((codes, scales)))
    shared, W = Q.new_codes(8, 24, "cpu"), torch.zeros(8, 24)
    for train in (True, False):
        lin = Q.Linear(4, 24, 8, torch.float32, train=train, device="cpu")
        lin.set_weight(*shared)
        assert lin.w_codes is shared[0] and lin.w_scales is shared[1]
        lin.pack_weight(W)
        own = seen[-1]
        assert own[0] is not shared[0] and own[1] is not shared[1] and lin.w_codes is own[0] and lin.w_scales is own[1]
        lin.set_weight(*shared)
        lin.pack_weight(W)
        assert seen[-1][0] is own[0] and seen[-1][1] is own[1]      # allocated once


def _held(*objects):
    """Bytes of the distinct buffers that objects hold, themselves or in what they are made of."""
    seen = {}

    def look(o):
        for v in vars(o).values():
            for t in v if isinstance(v, tuple) else (v,):
                if isinstance(t, torch.Tensor):
                    seen[t.untyped_storage().data_ptr()] = t.untyped_storage().nbytes()
                elif type(t).__module__ == type(o).__module__:
                    look(t)

    for o in objects:
        look(o)
    return sum(seen.values())


@pytest.mark.parametrize("M,C,F,dtype", [(1568, 64, 256, torch.bfloat16), (40, 72, 136, torch.float32), (4, 64, 96, torch.bfloat16)])
def test_a_further_block_of_a_stack_adds_codes_and_gradients_of_weights_only(M, C, F, dtype):
    """By the buffers that the objects hold: the full-width rows and the workspace are there once for the stack."""
    from paper_2305_11624_amd import quant as Q
    e = torch.finfo(dtype).bits // 8
    one = Q.GatedBlock(M, C, F, dtype, device="cpu")
    more = [Q.GatedBlock(M, C, F, dtype, device="cpu", share=one) for _ in range(3)]
    dW = 3 * F * C * e + 4 * (2 * F + C)      # and the biases' gradients
    assert _held(one, *more) - _held(one) == 3 * (one.saved_bytes() + dW)
    assert one.gate.dh is one.up.z            # h's gradient in h's place
    assert _held(one) == one.saved_bytes() + dW + e * M * (3 * F + 2 * C) + one.up.ws.nbytes
    assert one.up.ws is one.down.ws
    serve = [Q.GatedBlock(M, C, F, dtype, train=False, device="cpu", share=one) for _ in range(2)]
    assert _held(one, *serve) - _held(one) == 2 * M * (B.convbn_qrow_bytes(F) + 4)      # (y packed)
    for bad in (dict(M=M + 1), dict(C=C + 8), dict(F=F + 8), dict(dtype=torch.float32 if e == 2 else torch.bfloat16)):
        with pytest.raises(ValueError):
            Q.GatedBlock(**{**dict(M=M, C=C, F=F, dtype=dtype), **bad}, device="cpu", share=one)
    with pytest.raises(ValueError):
        Q.GatedBlock(M, C, F, dtype, device="cpu", share=serve[0])


def test_buffers_of_the_caller_and_gradients_that_are_not_asked_for():
    from paper_2305_11624_amd import quant as Q
    z, dx, ws = torch.zeros(40, 8), torch.zeros(40, 24), torch.zeros(Q.linear_workspace_bytes(40, 24, 8, torch.float32), dtype=torch.uint8)
    lin = Q.Linear(40, 24, 8, torch.float32, device="cpu", z=z, dx=dx, ws=ws)
    assert lin.z is z and lin.dx is dx and lin.ws is ws
    for bad in (dict(z=z.t()), dict(z=z[:-1]), dict(dx=dx.bfloat16()), dict(z=torch.zeros(40, 9)[:, :8]), dict(z=torch.zeros(40, 16)[:, ::2]), dict(ws=ws[:-1]),
                dict(z=torch.zeros(40, 8, device="meta"))):
        with pytest.raises(ValueError):
            Q.Linear(40, 24, 8, torch.float32, device="cpu", **bad)
    first = Q.Linear(40, 24, 8, torch.float32, device="cpu", need_dx=False)
    assert first.dx is None and first.dW is not None
    first.set_weight(*Q.new_codes(8, 24, "cpu"))
    with pytest.raises(RuntimeError):
        first.backward(torch.zeros(40, 8), need_dx=True)
    frozen = Q.Linear(40, 24, 8, torch.float32, device="cpu", need_dW=False)
    assert frozen.dW is None and frozen.dx is not None
    y, dh = torch.zeros(4, 8), torch.zeros(4, 16)
    gate = Q.Gate(4, 8, torch.float32, device="cpu", y=y, dh=dh)
    assert gate.y is y and gate.dh is dh
    out = torch.zeros(4, 8)
    assert Q.Checkpoint(4, 8, torch.float32, device="cpu", out=out).out is out
    for make in (lambda: Q.Gate(4, 8, torch.float32, device="cpu", y=y[:, :7]), lambda: Q.Gate(4, 8, torch.float32, device="cpu", dh=dh[:3]),
                 lambda: Q.Checkpoint(4, 8, torch.float32, device="cpu", out=out.bfloat16())):
        with pytest.raises(ValueError):
            make()


@pytest.mark.parametrize("train", [True, False])
def test_forward_of_no_tensor_is_refused(train, monkeypatch):
    """The entry point reads given codes where it gets no rows; a layer's forward has rows, and never multiplies what its buffers still hold."""
    from paper_2305_11624_amd import quant as Q
    monkeypatch.setattr(B, "convbn_qlinear_fwd", lambda *a: pytest.fail("launched"))
    lin = Q.Linear(4, 24, 8, torch.float32, train=train, device="cpu")
    lin.set_weight(*Q.new_codes(8, 24, "cpu"))
    with pytest.raises(ValueError):
        lin.forward(None)
    for codes, scales in ((None, None), (lin.w_codes, None)):
        with pytest.raises(ValueError):
            lin.forward_packed(codes, scales)
