"""Edges of the operators for a head on the GPU: every byte of kept 8-bit floating-point rows, group norm of values far from zero and behind an
outlying first value, infinite gradients behind a closed ReLU, what fp32 operands in parts leave out, infinite operands, a
stack on shared buffers, buffers that hold NaN before a call.

Bounds are those of head_ref.py, with U = 2^-24."""
import numpy as np
import pytest
import torch

from paper_2305_11624_amd import binding as B

import head_ref as R
from head_ref import DT, U, np64, within

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


# ---- what workspaces and outputs hold before a call ------------------------------------------------------------------

@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 20, 64, 300])
@pytest.mark.parametrize("F", [1, 2, 3, 4, 5, 6, 7, 8, 9, 29, 62, 70, 71, 261])
def test_gated_product_of_any_width_reads_nothing_that_it_has_not_written(F, M, dtype, keep):
    """Buffers full of NaN in front of each call change no bit."""
    from paper_2305_11624_amd import gated as G
    K, dt = 40, DT[dtype]
    x, W, dy = (torch.randn(*s, generator=R.gen(i)).to("cuda", dt) for i, s in enumerate([(M, K), (2 * F, K), (M, F)]))
    b = torch.randn(2 * F, generator=R.gen(4)).cuda()
    results = []
    for value in (0, 255):
        lay = G.Gated(M, K, F, dt, keep=keep)
        for t in (lay.ws, lay.h, lay.y, lay.dx, lay.dW, lay.db):
            if t is not None:
                t.view(torch.uint8).fill_(value)
        y = lay.forward(x, W, b).clone()
        if lay.ws is not None:
            lay.ws.fill_(value)
        results.append([y] + [t.clone() for t in lay.backward(x, W, dy, b)])
    assert all(torch.isfinite(a).all() and torch.equal(a, c) for a, c in zip(*results))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [1, 20, 300])
@pytest.mark.parametrize("K,N", [(1, 1), (3, 5), (40, 29), (130, 70), (300, 261), (513, 6), (129, 127)])
def test_f8_linear_of_any_width_reads_nothing_that_it_has_not_written(K, N, M, dtype):
    from paper_2305_11624_amd import quant as Q
    dt = DT[dtype]
    x, W, dz = (torch.randn(*s, generator=R.gen(i)).to("cuda", dt) for i, s in enumerate([(M, K), (N, K), (M, N)]))
    results = []
    for value in (0, 255):
        lay = Q.F8Linear(M, K, N, dt)
        lay.pack_weight(W)
        for t in (lay.w_codes, lay.w_scales, lay.codes, lay.scales, lay.ws, lay.z, lay.dx, lay.dW, lay.db):
            if t is not None:
                t.view(torch.uint8).fill_(value)
        lay.pack_weight(W)
        z = lay.forward(x).clone()
        if lay.ws is not None:
            lay.ws.fill_(value)
        results.append([z] + [t.clone() for t in lay.backward(dz, bias=True)])
    assert all(torch.isfinite(a).all() and torch.equal(a, c) for a, c in zip(*results))


# ---- group norm -----------------------------------------------------------------------------------------------------

# images, pixels, channels, groups: pieces of eight, with tails and single channels, in one launch and in segments
WALKS = [(2, 64, 64, 1), (3, 1, 4096, 1), (2, 300, 32, 4), (3, 100, 65, 1), (2, 33, 65, 5), (5, 891, 72, 8), (1, 30000, 16, 2), (2, 5000, 24, 3), (1, 2289, 1472, 1),
         (40, 9, 32, 4), (300, 1, 40, 1)]


def _norm_within(x, images, G, act, dtype, centre, params=True):
    """Forward and backward of x against the formulas on x - centre, a number for each group, which gives the same results, but with bounds
    that know nothing of the centre's size."""
    from paper_2305_11624_amd import norm as N
    C, dt = x.shape[1], DT[dtype]
    P = x.shape[0] // images
    ga, be = 1 + 0.3 * torch.randn(C, generator=R.gen(1)), 0.3 * torch.randn(C, generator=R.gen(2))
    dy = torch.randn(x.shape, generator=R.gen(3)).to(dt).float()
    lay = N.GroupNorm(images, P, C, G, dt, act=act)
    xd, gd, bd = x.to("cuda", dt), ga.cuda(), be.cuda()
    x64 = np64(xd).reshape(images, P, G, C // G)
    near = (x64 - centre(x64)).reshape(x.shape)
    want = R.norm(near, images, G, act, dtype, np64(ga), np64(be), 1e-5, np64(dy))
    within(lay.forward(xd, gd, bd), *want["y"], "y")
    dx, dgamma, dbeta = lay.backward(xd, gd, bd, dy.to("cuda", dt))
    within(dx, *want["dx"], "dx")
    within(dgamma, *want["dgamma"], "dgamma")
    within(dbeta, *want["dbeta"], "dbeta")


@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("first,rest", [(1e3, 0), (-1e5, 0), (0, 1e4)])
@pytest.mark.parametrize("images,P,C,G", WALKS)
def test_group_norm_behind_an_outlying_first_value(images, P, C, G, first, rest, act):
    """The first value of each group far from all others: a loud channel, a zero of padding in front of a map whose mean is not zero."""
    x = torch.randn(images, P, G, C // G, generator=R.gen(7)) + rest
    x[:, 0, :, 0] = first
    _norm_within(x.reshape(images * P, C), images, G, act, "f32", lambda v: np.median(v, axis=(1, 3), keepdims=True))


@pytest.mark.parametrize("dtype,mean", [("bf16", 200), ("f32", 1e4)])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("images,P,C,G", WALKS)
def test_group_norm_of_a_mean_far_from_zero(images, P, C, G, act, dtype, mean):
    """Results have the bits that the differences to the mean have, not those that the values leave."""
    x = torch.randn(images * P, C, generator=R.gen(8)) + mean
    _norm_within(x, images, G, act, dtype, lambda v: mean)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,P,C,G", [(2, 49, 64, 8), (300, 1, 40, 1), (2, 33, 65, 5), (1, 20000, 8, 1)])
def test_infinite_gradients_behind_a_closed_relu_are_none(images, P, C, G, dtype):
    from paper_2305_11624_amd import norm as N
    dt = DT[dtype]
    x, dy = (torch.randn(images * P, C, generator=R.gen(i)).to("cuda", dt) for i in (1, 2))
    lay = N.GroupNorm(images, P, C, G, dt, act="relu")
    closed = lay.forward(x) == 0
    results = []
    for v in (0.0, float("inf"), float("-inf"), float("nan")):
        d = torch.where(closed, torch.full_like(dy, v), dy)
        results.append([t.clone() for t in lay.backward(x, None, None, d)])
    for r in results:
        assert all(torch.isfinite(t).all() and torch.equal(t, z) for t, z in zip(r, results[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu"])
@pytest.mark.parametrize("images,P,C,G", WALKS)
def test_group_norm_reads_nothing_that_it_has_not_written(images, P, C, G, act, dtype):
    from paper_2305_11624_amd import norm as N
    dt = DT[dtype]
    x, dy = (torch.randn(images * P, C, generator=R.gen(i)).to("cuda", dt) for i in (1, 2))
    ga, be = (torch.randn(C, generator=R.gen(i)).cuda() for i in (3, 4))
    results = []
    for value in (0, 255):
        lay = N.GroupNorm(images, P, C, G, dt, act=act)
        for t in (lay.ws, lay.stats, lay.y, lay.dx, lay.dgamma, lay.dbeta):
            if t is not None:
                t.view(torch.uint8).fill_(value)
        y = lay.forward(x, ga, be).clone()
        if lay.ws is not None:
            lay.ws.fill_(value)
        results.append([y] + [t.clone() for t in lay.backward(x, ga, be, dy)])
    assert all(torch.isfinite(a).all() and torch.equal(a, c) for a, c in zip(*results))


# ---- fp32 operands of the gated product in parts --------------------------------------------------------------------

def _gated(M, K, F, dtype, **kw):
    from paper_2305_11624_amd import gated as G
    return G.Gated(M, K, F, DT[dtype], **kw)


def _shrinks(got, want):
    """The mean of what got lies nearer to zero than want, in units of U |want|."""
    got, want = np64(got), np64(want)
    return float((np.sign(want) * (want - got) / np.abs(want)).mean() / U)


@pytest.mark.parametrize("M,F", [(16, 4096), (300, 512)])
def test_products_of_fp32_numbers_in_parts_are_not_drawn_to_zero(M, F):
    """Products of one term each, of either sign.  What is left out of such a product, and each rounding of its sum, is at most some U of it and as often up as
    down: over 10^5 of them the mean is below 0.1 U (parts that are cut off rather than rounded make 0.7).  Either is at most 7 U in one."""
    x, W = (torch.randn(n, 1, generator=R.gen(n)) for n in (M, 2 * F))
    lay = _gated(M, 1, F, "f32")
    lay.forward(x.cuda(), W.cuda())
    want = x.double() @ W.double().T
    assert abs(_shrinks(lay.h.view(M, 2 * F), want)) < 0.1
    within(lay.h.view(M, 2 * F), np64(want), 12 * U * np.abs(np64(want)), "h")


def test_gradients_of_fp32_numbers_in_parts_are_not_drawn_to_zero():
    """One row: db is dh, and each number of dW one product of it."""
    K, F = 700, 600
    x, W = torch.randn(1, K, generator=R.gen(1)), torch.randn(2 * F, K, generator=R.gen(2)) * K ** -0.5
    lay = _gated(1, K, F, "f32")
    b, dy = torch.zeros(2 * F, device="cuda"), torch.randn(1, F, generator=R.gen(3)).cuda()
    lay.forward(x.cuda(), W.cuda(), b)
    _, dW, db = lay.backward(x.cuda(), W.cuda(), dy, b)
    want = db.cpu().double()[:, None] * x.double()
    assert abs(_shrinks(dW, want)) < 0.1
    within(dW, np64(want), 12 * U * np.abs(np64(want)), "dW")


@pytest.mark.parametrize("M", [2, 40])
def test_largest_fp32_numbers_in_parts_stay_finite(M):
    """Numbers above bf16's largest, and fp32's largest itself: one term each, so that what is left out and six roundings are at most 7 U of it."""
    x = torch.tensor([torch.finfo(torch.float32).max, -3.4e38]).repeat(M // 2)[:, None]
    W = torch.tensor([0.5, -0.25, 1 / 3, 0.9])[:, None]
    lay = _gated(M, 1, 2, "f32")
    lay.forward(x.cuda(), W.cuda())
    want = np64(x) @ np64(W).T
    within(lay.h.view(M, 4), want, 7 * U * np.abs(want), "h")


def _same_kind(got, want, name):
    """Infinities of the same sign, NaN, and finite numbers in the same places."""
    got, want = np64(got), np.asarray(want)
    for kind in (np.isnan, np.isposinf, np.isneginf):
        assert np.array_equal(kind(got), kind(want)), (name, kind.__name__)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M", [3, 70])
def test_infinite_operands_of_the_gated_product(M, dtype):
    """An infinity meets numbers that bf16 holds (whose lower parts are zero), others, and a zero."""
    K, F, dt = 40, 24, DT[dtype]
    x, W = torch.randn(M, K, generator=R.gen(1)).to(dt).float(), torch.randn(2 * F, K, generator=R.gen(2)).to(dt).float()
    W[::2] = W[::2].bfloat16().float()
    x[::2] = x[::2].bfloat16().float()
    x[0, 3], x[1, 39], x[2, 5] = float("inf"), float("-inf"), 0
    W[7, 5], W[30, 11], W[4, 3] = float("inf"), float("-inf"), 0
    lay = _gated(M, K, F, dtype)
    lay.forward(x.to("cuda", dt), W.to("cuda", dt))
    with np.errstate(invalid="ignore"):
        _same_kind(lay.h.view(M, 2 * F), np64(x) @ np64(W).T, "h")


@pytest.mark.parametrize("M", [3, 70])
def test_infinite_gradients_of_the_gated_product(M):
    K, F = 40, 24
    x, W = torch.randn(M, K, generator=R.gen(1)), torch.randn(2 * F, K, generator=R.gen(2)) * K ** -0.5
    x[::2], W[::2] = x[::2].bfloat16().float(), W[::2].bfloat16().float()
    dy = torch.randn(M, F, generator=R.gen(3))
    dy[1, 4], dy[2, 9] = float("inf"), float("-inf")
    lay = _gated(M, K, F, "f32")
    b = torch.zeros(2 * F)
    lay.forward(x.cuda(), W.cuda(), b.cuda())
    dx, dW, db = lay.backward(x.cuda(), W.cuda(), dy.cuda(), b.cuda())
    with np.errstate(invalid="ignore"):
        h = np64(x) @ np64(W).T
        f, df, _ = R.act("silu", h[:, :F])
        dh = np.concatenate([np64(dy) * h[:, F:] * df, np64(dy) * f], 1)
        _same_kind(db, dh.sum(0), "db")
        _same_kind(dx, dh @ np64(W), "dx")
        _same_kind(dW, dh.T @ np64(x), "dW")


# ---- a stack ---------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("images,P,C,F,G", [(2, 49, 64, 136, 8), (1, 20000, 8, 24, 1), (300, 1, 72, 40, 1)])
def test_gradient_of_a_stack_on_shared_buffers(images, P, C, F, G):
    """Three blocks on one set of buffers: each block's gradient is handed on as it comes, in the buffer that the next one writes, and gives what blocks with
    buffers of their own give."""
    from paper_2305_11624_amd.gated import NormGatedBlock
    g = R.gen(11)
    dt = torch.bfloat16
    x, dout = (torch.randn(images * P, C, generator=g).to("cuda", dt) for _ in range(2))
    Wu = (torch.randn(2 * F, C, generator=g) * C ** -0.5).to("cuda", dt)
    Wd = (torch.randn(C, F, generator=g) * F ** -0.5).to("cuda", dt)
    ga, be = (1 + 0.2 * torch.randn(C, generator=g)).cuda(), (0.2 * torch.randn(C, generator=g)).cuda()
    results = []
    for shared in (False, True):
        blocks = [NormGatedBlock(images, P, C, F, G, dt)]
        blocks += [NormGatedBlock(images, P, C, F, G, dt, share=blocks[0] if shared else None) for _ in range(2)]
        assert not shared or len({b.norm.dx.data_ptr() for b in blocks}) == 1
        ins, v = [], x
        for b in blocks:
            b.pack_weight(Wd)
            ins.append(v)
            v = b.forward(v, Wu, ga, be)
        found, d = [v.clone()], dout
        for b, i in zip(blocks[::-1], ins[::-1]):
            d, *params = b.backward(i, Wu, ga, be, d)
            found += [t.clone() for t in params]
        results.append(found + [d.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*results))


# ---- more than 2^31 elements -------------------------------------------------------------------------------------------

def _some_rows(M):
    return [0, 1, M // 2, M - 2, M - 1]


def test_group_norm_of_tokens_past_2_31_elements():
    """The last tokens like the first: what a layer of these tokens alone gives.  dy is zero but for them, so that dgamma and dbeta are theirs."""
    from paper_2305_11624_amd import norm as N
    C, dt = 4104, torch.bfloat16
    M = (1 << 31) // C + 7
    some = _some_rows(M)
    x, dy = torch.zeros(M, C, dtype=dt, device="cuda"), torch.zeros(M, C, dtype=dt, device="cuda")
    rows = [torch.randn(len(some), C, generator=R.gen(i)).to("cuda", dt) for i in (1, 2)]
    x[some], dy[some] = rows
    ga, be = (1 + 0.3 * torch.randn(C, generator=R.gen(3))).cuda(), (0.3 * torch.randn(C, generator=R.gen(4))).cuda()
    big, small = (N.GroupNorm(n, 1, C, 1, dt, act="silu") for n in (M, len(some)))
    assert torch.equal(big.forward(x, ga, be)[some], small.forward(rows[0], ga, be))
    dx, dgamma, dbeta = big.backward(x, ga, be, dy)
    want = small.backward(rows[0], ga, be, rows[1])
    assert torch.equal(dx[some], want[0])
    for got, ref in ((dgamma, want[1]), (dbeta, want[2])):      # (five terms, added in another order)
        assert ((got - ref).abs() <= 16 * U * (rows[1].float().abs() * 6).sum(0)).all()


def test_group_norm_of_an_image_past_2_31_elements():
    """Values +-1 in equal number, but for a last pixel of another kind: mean 0 and variance 1 to 2^-18."""
    from paper_2305_11624_amd import norm as N
    C, dt = 2056, torch.bfloat16
    P = (1 << 31) // C + 8
    x = torch.ones(P, C, dtype=dt, device="cuda")
    x[1::2] = -1
    x[-1], x[-2] = 2.0, -2.0
    lay = N.GroupNorm(1, P, C, 2, dt)
    y = lay.forward(x)
    for row in _some_rows(P):
        assert torch.equal(y[row], x[row]), row      # (bf16: half a step is 2^-9)
    dy = torch.zeros_like(x)
    dy[-1, -1] = 1.0
    dx, dgamma, dbeta = lay.backward(x, None, None, dy)
    assert float(dx[-1, -1]) == 1.0 and float(dgamma[-1]) == pytest.approx(2.0, rel=1e-4) and float(dbeta[-1]) == 1.0
    assert not dgamma[:-1].any() and not dbeta[:-1].any()


def test_f8_rows_past_2_31_elements():
    from paper_2305_11624_amd import quant as Q
    K, dt = 4104, torch.bfloat16
    M = (1 << 31) // K + 7
    some = _some_rows(M)
    x = torch.zeros(M, K, dtype=dt, device="cuda")
    x[some] = rows = torch.randn(len(some), K, generator=R.gen(1)).to("cuda", dt)
    big, small = Q.F8Checkpoint(M, K, dt), Q.F8Checkpoint(len(some), K, dt)
    big.pack(x)
    small.pack(rows)
    assert torch.equal(big.codes[some], small.codes) and torch.equal(big.scales[some], small.scales)
    out = big.unpack(x.fill_(3))
    assert torch.equal(out[some], small.unpack()) and not out[2:M // 2].any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_products_of_rows_that_lie_past_2_31_elements(dtype):
    """Rows 2^20 (read in place, where they can be) and 2^21 elements apart, 2^31 of them in all: the bits of rows next to each other."""
    from paper_2305_11624_amd import quant as Q
    dt, K, F = DT[dtype], 64, 48
    for M, ld in ((2100, 1 << 20), (1030, 1 << 21)):
        x, dy = (torch.randn(M, n, generator=R.gen(n)).to("cuda", dt) for n in (K, F))
        W = torch.randn(2 * F, K, generator=R.gen(1)).to("cuda", dt)
        buf = [torch.empty(M * ld, dtype=dt, device="cuda") for _ in range(2)]      # of inputs and of outputs: x and dy, y and dx side by side
        far = lambda i, at, n: buf[i].as_strided((M, n), (ld, 1), at)
        xf, dyf, yf, dxf = far(0, 0, K), far(0, 4096, F), far(1, 0, F), far(1, 4096, K)
        xf.copy_(x)
        dyf.copy_(dy)
        near = _gated(M, K, F, dtype)
        want = [near.forward(x, W).clone()] + [t.clone() for t in near.backward(x, W, dy)[:2]]
        lay = _gated(M, K, F, dtype)
        lay.desc.ldx = lay._add_desc.ldx = lay.desc.ldz = lay._add_desc.ldz = ld
        lay.y, lay.dx = yf, dxf
        lay.ws = torch.empty(max(B.convbn_glu_workspace_bytes(lay.desc, p) for p in (B.PASS_FWD, B.PASS_BWD)), dtype=torch.uint8, device="cuda")
        got = [lay.forward(xf, W).clone()] + [t.clone() for t in lay.backward(xf, W, dyf)[:2]]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), ld
        near = Q.F8Linear(M, K, F, dt)
        near.pack_weight(W[:F])
        want = [near.forward(x).clone()] + [t.clone() for t in near.backward(dy)[:2]]
        lay = Q.F8Linear(M, K, F, dt)
        lay.ldx = lay.ldz = lay.desc.ldx = lay.desc.ldz = lay._add_desc.ldx = lay._add_desc.ldz = ld
        lay.z, lay.dx = yf, dxf
        lay.ws = torch.empty(max(B.convbn_flinear_workspace_bytes(lay.desc, p) for p in (B.PASS_FWD, B.PASS_BWD)), dtype=torch.uint8, device="cuda")
        lay.pack_weight(W[:F])
        got = [lay.forward(xf).clone()] + [t.clone() for t in lay.backward(dyf)[:2]]
        assert all(torch.equal(a, b) for a, b in zip(got, want)), ld
        del buf
