"""The operators for a head on the GPU against plain implementations in 64 bits: rows in 8-bit floating point and their product, the gated
product, group norm, and a block of the three.

Two kinds of comparison.  Exact: where the values are small whole numbers every sum fits 24 bits, and the result has to be the exact one,
rounded once.  Bounded: elsewhere an output may be off by what the stated roundings allow, element by element (head_ref.py; with U = 2^-24 and
R summed terms t, (R + 8) U sum |t| for a sum, half a step for a rounding)."""
import numpy as np
import pytest
import torch

from paper_2305_11624_amd import binding as B

import head_ref as R
from head_ref import DT, U, half, np64, on_device, within

pytestmark = pytest.mark.gpu


def _mods():
    from paper_2305_11624_amd import gated, norm, quant
    return quant, gated, norm


def _whole(rows, K, seed, most=8):
    """Whole numbers that e4m3 holds whatever the scale of their block."""
    return torch.randint(-most, most + 1, (rows, K), generator=R.gen(seed)).float()


def _tokens(M, K, dt, seed, loud=9):
    x = torch.randn(M, K, generator=R.gen(seed))
    x[:, ::17] *= loud
    if M > 2:
        x[M // 2] = 0
    return x.to(dt).float()


# ---- 8-bit floating point: rows ------------------------------------------------------------------------------------

ROWS = [(1, 1), (2, 7), (3, 16), (5, 127), (4, 128), (4, 129), (7, 255), (9, 256), (3, 512), (3, 513), (2, 1000), (2, 4100), (1, 8200), (700, 24)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [0, 8, 5])
@pytest.mark.parametrize("M,K", ROWS)
def test_f8_pack_and_unpack(M, K, gap, dtype):
    Q, dt = _mods()[0], DT[dtype]
    x = _tokens(M, K, dt, M * 1000 + K)
    ck = Q.F8Checkpoint(M, K, dt)
    ck.codes.fill_(77)
    ck.scales.fill_(3)
    ck.pack(on_device(x, gap, dt))
    q, s = R.f8_pack(x)
    got, gs = ck.codes.cpu().numpy(), ck.scales.cpu().numpy()
    assert np.array_equal(gs[:, :s.shape[1]], s) and (gs[:, s.shape[1]:] == 127).all()
    assert np.array_equal(got[:, :K], q) and (got[:, K:] == 0).all()
    out = on_device(torch.zeros(M, K), gap, dt)
    ck.unpack(out)
    assert np.array_equal(np64(out), R.f8_values(q, s))      # (exact: a bf16 number)
    if gap and M > 1:
        assert torch.isnan(out.as_strided((M - 1, gap), (out.stride(0), 1), K)).all()      # nothing between the rows


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_f8_pack_special_blocks(dtype):
    Q, dt = _mods()[0], DT[dtype]
    K, big = 300, torch.finfo(dt).max
    x = torch.randn(14, K, generator=R.gen(5))
    x[0] = 0
    x[1] *= 2.0 ** -126                               # below the smallest block that keeps all bits
    x[2] *= 2.0 ** -140
    x[3, 130] = float("inf")
    x[4, 299] = float("nan")
    x[5, 0], x[5, 1] = big, -big
    x[6, 129] = -big                                   # a mask's lowest value in front of small ones
    every = torch.from_numpy(R.e4m3_values()[:127]).float()
    x[7, :127], x[7, 127] = every, 0                   # every code at the scale 1
    x[8, :126] = (every[1:] + every[:-1]) / 2          # and the ties between them
    x[8, 126], x[8, 127] = 448, -432
    x[9, :128] = 2.0 ** 120
    x[10, :128] = 448 * 2.0 ** 3                       # at the border of a scale, and just past it
    x[11, :128] = 449 * 2.0 ** 3
    x[12] = 2.0 ** -133
    x[13] = -0.0
    x = x.to(dt).float()
    ck = Q.F8Checkpoint(14, K, dt)
    ck.pack(x.to("cuda", dt))
    q, s = R.f8_pack(x)
    assert np.array_equal(ck.scales.cpu().numpy()[:, :3], s)
    got = ck.codes.cpu().numpy()[:, :K]
    bad = np.isnan(R.f8_values(q, s))
    assert np.array_equal(got & np.where(bad, 127, 255), q & np.where(bad, 127, 255))
    back = np64(ck.unpack())
    assert np.array_equal(back, R.f8_values(q, s), equal_nan=True)
    assert np.isnan(back[3, 128:256]).all() and np.isfinite(back[3, :128]).all() and np.isfinite(back[[0, 1, 2, 5, 6, 9]]).all()


# ---- 8-bit floating point: products --------------------------------------------------------------------------------

# rows, channels in and out: single tokens, tile borders, every tail of a chunk, one channel, long sums, tall and wide
MULS = [(1, 1, 1), (1, 2048, 96), (2, 130, 33), (5, 64, 8), (8, 512, 257), (17, 100, 64), (31, 1025, 40), (33, 128, 129), (64, 640, 70),
        (65, 72, 136), (130, 260, 300), (257, 384, 64), (300, 4097, 48), (777, 136, 72), (1, 9000, 24), (40, 16, 1500), (1500, 24, 16)]


def _largest_of_eight(x8, w8):
    """The sum over groups of eight neighbouring channels of each group's largest product: the instruction for these codes keeps 13 bits below
    that one's leading bit, so each of the other seven loses less than 2^-13 of it."""
    pad = -x8.shape[1] % 8
    a, b = (np.abs(np.pad(v, ((0, 0), (0, pad)))).reshape(v.shape[0], -1, 8) for v in (x8, w8))
    return np.stack([(row[None] * b).max(axis=2).sum(axis=1) for row in a])


def _f8_layer(M, K, N, dtype, gap=0, train=True, **kw):
    return _mods()[0].F8Linear(M, K, N, DT[dtype], train=train, gap=gap, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gap", [0, 5])
@pytest.mark.parametrize("M,K,N", MULS)
def test_f8_linear_of_whole_numbers_is_exact(M, K, N, gap, dtype):
    dt = DT[dtype]
    x, W, dz, b, add, addx = (_whole(*s, 7 * M + K + N + i, m) for i, (s, m) in enumerate(
        [((M, K), 8), ((N, K), 8), ((M, N), 3), ((1, N), 100), ((M, N), 50), ((M, K), 50)]))
    lay = _f8_layer(M, K, N, dtype, gap)
    lay.pack_weight(W.to("cuda", dt))
    z = lay.forward(on_device(x, gap, dt), b[0].cuda(), add=on_device(add, gap, dt))
    want = x.double() @ W.double().T + b.double() + add.double()
    assert torch.equal(z.cpu(), want.float().to(dt))
    dx, dW, db = lay.backward(on_device(dz, gap, dt), bias=True, add=on_device(addx, gap, dt))
    assert torch.equal(dx.cpu(), (dz.double() @ W.double() + addx.double()).float().to(dt))
    assert torch.equal(dW.cpu(), (dz.double().T @ x.double()).float().to(dt))
    assert torch.equal(db.cpu(), dz.sum(0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", MULS)
def test_f8_linear_within_its_roundings(M, K, N, dtype):
    dt, hs = DT[dtype], half(dtype)
    x, W = _tokens(M, K, dt, M + K), (torch.randn(N, K, generator=R.gen(N)) * K ** -0.5).to(dt).float()
    x[:, K // 3] *= 300                                # a loud channel: its block's scale is another
    x = x.to(dt).float()
    dz = (1e-3 * torch.randn(M, N, generator=R.gen(3))).to(dt).float()
    lay = _f8_layer(M, K, N, dtype)
    lay.pack_weight(W.to("cuda", dt))
    z = lay.forward(x.to("cuda", dt))
    x8, w8 = R.f8_values(*R.f8_pack(x)), R.f8_values(*R.f8_pack(W))
    want, mag = x8 @ w8.T, np.abs(x8) @ np.abs(w8).T
    e = (K + 8) * U * mag + (7 * 2.0 ** -13 * _largest_of_eight(x8, w8) if dtype == "bf16" else 0)
    within(z, want, e + hs * (np.abs(want) + e), "z")
    dx, dW, db = lay.backward(dz.to("cuda", dt), bias=True)
    d = dz.double().numpy()
    for got, want, mag, n, name in ((dx, d @ w8, np.abs(d) @ np.abs(w8), N, "dx"), (dW, d.T @ x8, np.abs(d).T @ np.abs(x8), M, "dW")):
        e = (n + 8) * U * mag
        within(got, want, e + hs * (np.abs(want) + e), name)
    within(db, d.sum(0), (M + 8) * U * np.abs(d).sum(0), "db")


@pytest.mark.parametrize("M", [1, 40, 300])
def test_f8_serving_reads_given_codes_and_keeps_none(M):
    Q = _mods()[0]
    K, N = 400, 200
    x, W = _whole(M, K, 1), _whole(N, K, 2)
    w = Q.new_f8_codes(N, K)
    B.convbn_fpack(B.make_qdesc(N, K), W.to("cuda", torch.bfloat16), *w)
    before = [t.clone() for t in w]
    lay = _f8_layer(M, K, N, "bf16", train=False)
    lay.set_weight(*w)
    z = lay.forward(x.to("cuda", torch.bfloat16)).clone()
    assert torch.equal(z.float().cpu(), (x @ W.T).bfloat16().float())
    codes = Q.new_f8_codes(M, K)
    B.convbn_fpack(B.make_qdesc(M, K), x.to("cuda", torch.bfloat16), *codes)
    assert torch.equal(lay.forward_packed(*codes), z)
    assert all(torch.equal(a, b) for a, b in zip(before, w)) and lay.saved_bytes() == 0


def test_f8_special_rows_stay_in_their_rows():
    M, K, N = 70, 300, 40
    x, W = torch.randn(M, K, generator=R.gen(1)), torch.randn(N, K, generator=R.gen(2))
    x[3, 10], x[5, 299], x[7] = float("nan"), float("inf"), 0
    lay = _f8_layer(M, K, N, "f32")
    lay.pack_weight(W.cuda())
    z = lay.forward(x.cuda()).cpu()
    assert torch.isnan(z[[3, 5]]).all() and (z[7] == 0).all()
    keep = [m for m in range(M) if m not in (3, 5)]
    assert torch.isfinite(z[keep]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_f8_no_rows(dtype):
    lay = _f8_layer(0, 64, 32, dtype)
    lay.pack_weight(torch.ones(32, 64, device="cuda", dtype=DT[dtype]))
    x, dz = (torch.empty(0, n, device="cuda", dtype=DT[dtype]) for n in (64, 32))
    assert lay.forward(x).shape == (0, 32)
    lay.dW.fill_(7)
    lay.db.fill_(7)
    dx, dW, db = lay.backward(dz, bias=True)
    assert dx.shape == (0, 64) and (dW == 0).all() and (db == 0).all()


# ---- gated product -------------------------------------------------------------------------------------------------

GLUS = [(1, 1, 1), (1, 2048, 96), (2, 130, 33), (5, 64, 8), (8, 512, 257), (16, 72, 40), (17, 100, 64), (33, 128, 129), (64, 640, 70),
        (130, 264, 300), (257, 384, 64), (300, 2051, 48), (777, 136, 72), (40, 16, 1500), (1500, 24, 16)]


def _glu_case(M, K, F, dtype, seed):
    dt = DT[dtype]
    x = _tokens(M, K, dt, seed, 3)
    W = (torch.randn(2 * F, K, generator=R.gen(seed + 1)) * K ** -0.5).to(dt).float()
    b = torch.randn(2 * F, generator=R.gen(seed + 2))
    dy = (1e-2 * torch.randn(M, F, generator=R.gen(seed + 3))).to(dt).float()
    return x, W, b, dy


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("kind,bias,gap", [("silu", False, 0), ("gelu", True, 5)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,F", GLUS)
def test_gated_product(M, K, F, dtype, kind, bias, gap, keep):
    G, dt = _mods()[1], DT[dtype]
    x, W, b, dy = _glu_case(M, K, F, dtype, M + K + F)
    add = _whole(M, K, 4, 2)
    lay = G.Gated(M, K, F, dt, kind, keep=keep, gap=gap)
    xd, Wd, bd, dyd = on_device(x, gap, dt), W.to("cuda", dt), b.cuda() if bias else None, on_device(dy, gap, dt)
    y = lay.forward(xd, Wd, bd)
    dx, dW, db = lay.backward(xd, Wd, dyd, bd, add=on_device(add, gap, dt))
    want = R.gated(*(np64(t) for t in (x, W)), np64(b) if bias else None, kind, dtype, np64(dy), np64(add))
    within(y, *want["y"], "y")
    within(dx, *want["dx"], "dx")
    within(dW, *want["dW"], "dW")
    if bias:
        within(db, *want["db"], "db")
    else:
        assert db is None


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gated_product_gives_what_is_asked_for(dtype):
    G, dt = _mods()[1], DT[dtype]
    M, K, F = 200, 136, 72
    x, W, b, dy = (t.to("cuda", dt) for t in _glu_case(M, K, F, dtype, 9))
    b = b.float()
    lay = G.Gated(M, K, F, dt)
    lay.forward(x, W, b)
    full = [t.clone() for t in lay.backward(x, W, dy, b)]
    for need_dx, need_dW, bias in [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 1, 1), (1, 1, 0)]:
        for t in (lay.dx, lay.dW, lay.db):
            t.fill_(7)
        st = B.convbn_glu_bwd(lay.desc, x, W, b, lay.h, dy, lay.dx if need_dx else None, lay.dW if need_dW else None, lay.db if bias else None, lay.ws)
        assert st == B.OK
        for got, want, asked in zip((lay.dx, lay.dW, lay.db), full, (need_dx, need_dW, bias)):
            assert torch.equal(got, want) if asked else (got == 7).all()


def test_gated_product_no_rows_and_special_rows():
    G = _mods()[1]
    lay = G.Gated(0, 64, 32, torch.float32)
    W = torch.randn(64, 64, device="cuda")
    b = torch.zeros(64, device="cuda")
    x, dy = (torch.empty(0, n, device="cuda") for n in (64, 32))
    assert lay.forward(x, W, b).shape == (0, 32)
    dx, dW, db = lay.backward(x, W, dy, b)
    assert (dW == 0).all() and (db == 0).all()
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn(70, 64, device="cuda").to(dt)
        x[3, 5], x[9, 63] = float("nan"), float("inf")
        y = G.Gated(70, 64, 32, dt, train=False).forward(x, W.to(dt)).float()
        keep = [m for m in range(70) if m not in (3, 9)]
        assert torch.isnan(y[3]).all() and not torch.isfinite(y[9]).all() and torch.isfinite(y[keep]).all()


def _difference(f, at, along, eps):
    return (f(at + eps * along) - f(at - eps * along)) / (2 * eps)


@pytest.mark.parametrize("keep", [True, False])
def test_gated_gradients_against_differences(keep):
    """Along random directions, fp32.  eps = 2^-6: the difference is off by some eps^2 / 6 of a third derivative (of order 1 here) and by the
    rounding of y, some K U |y| |dy| sqrt(M F) / eps: both below 2e-3 of sums of this size."""
    G = _mods()[1]
    M, K, F = 33, 40, 24
    x, W, b, dy = (t.cuda() for t in _glu_case(M, K, F, "f32", 5))
    lay = G.Gated(M, K, F, torch.float32, "gelu", keep=keep)
    lay.forward(x, W, b)
    dx, dW, db = (t.clone() for t in lay.backward(x, W, dy, b))
    J = lambda x, W, b: float((lay.forward(x, W, b).double() * dy.double()).sum())
    for i, (t, g) in enumerate(((x, dx), (W, dW), (b, db))):
        v = torch.randn(t.shape, generator=R.gen(i)).cuda()
        args = [x, W, b]

        def f(a):
            args[i] = a
            return J(*args)

        slope = float((g.double() * v.double()).sum())
        size = float((g.double() * v.double()).norm()) * 4 + 1e-3
        assert abs(_difference(f, t, v, 2.0 ** -6) - slope) <= 2e-2 * size, i


# ---- group norm ----------------------------------------------------------------------------------------------------

# images, pixels, channels, groups
NORMS = [(1, 1, 64, 1), (3, 49, 64, 8), (2, 7, 72, 8), (1, 49, 2048, 32), (2, 196, 256, 32), (5, 891, 72, 8), (2, 64, 12, 12), (3, 100, 65, 1), (2, 33, 65, 5),
         (300, 1, 40, 1), (7, 1, 513, 1), (5, 1, 4096, 1), (3, 1, 4100, 2), (2, 1, 20001, 1), (1, 3136, 64, 2), (2, 5000, 24, 3), (1, 20000, 8, 1), (1, 4, 9000, 9),
         (1, 900, 192, 1), (40, 9, 32, 4), (1, 5000, 260, 26)]


def _norm_case(images, P, C, dtype, seed):
    dt = DT[dtype]
    x = (torch.randn(images * P, C, generator=R.gen(seed)) * (0.5 + torch.rand(C, generator=R.gen(seed + 1))) + 2 * torch.randn(C, generator=R.gen(seed + 2)))
    ga, be = 1 + 0.3 * torch.randn(C, generator=R.gen(seed + 3)), 0.3 * torch.randn(C, generator=R.gen(seed + 4))
    dy = 1e-2 * torch.randn(images * P, C, generator=R.gen(seed + 5))
    return x.to(dt).float(), ga, be, dy.to(dt).float()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act,gap,affine", [("none", 0, True), ("relu", 8, True), ("silu", 5, True), ("gelu", 0, False)])
@pytest.mark.parametrize("images,P,C,G", NORMS)
def test_group_norm(images, P, C, G, act, gap, affine, dtype):
    N, dt = _mods()[2], DT[dtype]
    x, ga, be, dy = _norm_case(images, P, C, dtype, images + P + C)
    lay = N.GroupNorm(images, P, C, G, dt, act=act, gap=gap)
    xd, dyd = on_device(x, gap, dt), on_device(dy, gap, dt)
    gd, bd = (ga.cuda(), be.cuda()) if affine else (None, None)
    want = R.norm(np64(x), images, G, act, dtype, np64(ga) if affine else None, np64(be) if affine else None, 1e-5, np64(dy))
    y = lay.forward(xd, gd, bd)
    within(y, *want["y"], "y")
    stats = lay.stats.view(-1, 4).double()      # each as a number and what it leaves
    within(stats[:, 0] + stats[:, 1], *want["mean"], "mean")
    within(stats[:, 2] + stats[:, 3], *want["rstd"], "rstd")
    dx, dgamma, dbeta = lay.backward(xd, gd, bd, dyd)
    for got, name in ((dx, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
        within(got, *want[name], name)
    if gap and images * P > 1:      # nothing between the rows (torch.empty: the gap of y and dx is the library's to leave alone)
        lay.y.as_strided((images * P - 1, gap), (C + gap, 1), C).fill_(3)
        lay.forward(xd, gd, bd)
        assert (lay.y.as_strided((images * P - 1, gap), (C + gap, 1), C) == 3).all()
    serve = N.GroupNorm(images, P, C, G, dt, act=act, gap=gap, train=False)
    assert torch.equal(serve.forward(xd, gd, bd), y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,P,C,G", [(3, 49, 64, 8), (9, 1, 520, 1), (2, 5000, 24, 3)])
def test_group_norm_addend_and_single_outputs(images, P, C, G, dtype):
    N, dt = _mods()[2], DT[dtype]
    x, ga, be, dy = _norm_case(images, P, C, dtype, 3)
    add = _whole(images * P, C, 8, 3)
    lay = N.GroupNorm(images, P, C, G, dt, act="silu")
    args = [t.to("cuda", dt) for t in (x, dy)]
    lay.forward(args[0], ga.cuda(), be.cuda())
    want = R.norm(np64(x), images, G, "silu", dtype, np64(ga), np64(be), 1e-5, np64(dy), np64(add))
    full = [t.clone() for t in lay.backward(args[0], ga.cuda(), be.cuda(), args[1], add=add.to("cuda", dt))]
    within(full[0], *want["dx"], "dx")
    lay.dx.copy_(add.to("cuda", dt))
    again = lay.backward(args[0], ga.cuda(), be.cuda(), args[1], add=lay.dx)      # in place
    assert all(torch.equal(a, b) for a, b in zip(again, full))
    for dx, params in ((True, False), (False, True)):
        for t in (lay.dx, lay.dgamma, lay.dbeta):
            t.fill_(7)
        got = lay.backward(args[0], ga.cuda(), be.cuda(), args[1], need_dx=dx, need_params=params)
        assert (got[0] is None) != dx and (got[1] is None) != params
        assert (lay.dx == 7).all() if not dx else True
        if params:
            assert torch.equal(lay.dgamma, full[1]) and torch.equal(lay.dbeta, full[2])
        else:
            assert (lay.dgamma == 7).all() and (lay.dbeta == 7).all()


def test_group_norm_constant_groups_special_values_and_no_images():
    N = _mods()[2]
    for dt in (torch.bfloat16, torch.float32):
        x = torch.randn(4 * 30, 32, generator=R.gen(1)).to("cuda", dt)
        x[:30, :8] = 3                                    # var = 0: xhat = 0, y = f(beta)
        x[30, 9] = float("nan")
        x[60, 17] = float("inf")
        be = torch.randn(32, device="cuda")
        lay = N.GroupNorm(4, 30, 32, 4, dt)
        y = lay.forward(x, None, be).float().view(4, 30, 4, 8)
        assert torch.equal(y[0, :, 0], be[:8].to(dt).float().expand(30, 8))
        assert torch.isnan(y[1, :, 1]).all() and torch.isnan(y[2, :, 2]).all()
        y[1, :, 1] = y[2, :, 2] = 0
        assert torch.isfinite(y).all()
        none = N.GroupNorm(0, 30, 32, 4, dt)
        e = torch.empty(0, 32, dtype=dt, device="cuda")
        assert none.forward(e).shape == (0, 32)
        none.dgamma.fill_(7)
        dx, dg, db = none.backward(e, None, None, e)
        assert (dg == 0).all() and (db == 0).all()


def test_group_norm_of_values_far_from_zero():
    """A mean a thousand deviations from zero: the variance comes from differences, or it would lose all of its bits."""
    N = _mods()[2]
    for images, P, C, G in ((2, 300, 32, 4), (3, 1, 1024, 1), (1, 30000, 16, 2)):
        x = (torch.randn(images * P, C, generator=R.gen(2)) + 1000).float()
        lay = N.GroupNorm(images, P, C, G, torch.float32)
        y = lay.forward(x.cuda())
        within(y, *R.norm(np64(x), images, G, "none", "f32")["y"], "y")


def test_group_norm_gradients_against_differences():
    N = _mods()[2]
    images, P, C, G = 2, 25, 24, 3
    x, ga, be, dy = (t.cuda() for t in _norm_case(images, P, C, "f32", 5))
    lay = N.GroupNorm(images, P, C, G, torch.float32, act="gelu")
    lay.forward(x, ga, be)
    grads = [t.clone() for t in lay.backward(x, ga, be, dy)]
    for i in range(3):
        v = torch.randn([x, ga, be][i].shape, generator=R.gen(i)).cuda()
        args = [x, ga, be]

        def f(a):
            args[i] = a
            return float((lay.forward(*args).double() * dy.double()).sum())

        slope = float((grads[i].double() * v.double()).sum())
        size = float((grads[i].double() * v.double()).norm()) * 4 + 1e-3
        assert abs(_difference(f, [x, ga, be][i], v, 2.0 ** -6) - slope) <= 2e-2 * size, i


# ---- together ------------------------------------------------------------------------------------------------------

def _block(images, P, C, F, groups, dt, **kw):
    return _mods()[1].NormGatedBlock(images, P, C, F, groups, dt, **kw)


def _block_inputs(images, P, C, F, dt):
    g = R.gen(11)
    x = torch.randn(images * P, C, generator=g).to("cuda", dt)
    ws = [(torch.randn(*s, generator=g) * s[1] ** -0.5).to("cuda", dt) for s in ((2 * F, C), (C, F))]
    ga, be = (1 + 0.2 * torch.randn(C, generator=g)).cuda(), (0.2 * torch.randn(C, generator=g)).cuda()
    dout = (1e-2 * torch.randn(images * P, C, generator=g)).to("cuda", dt)
    return x, *ws, ga, be, dout


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("images,P,C,F,groups", [(1, 1, 64, 128, 1), (40, 1, 72, 200, 1), (3, 49, 128, 264, 8)])
def test_block_is_its_parts(images, P, C, F, groups, keep):
    """fp32: every part against the plain form of its own inputs, and the whole within the 8-bit rounding of y."""
    blk = _block(images, P, C, F, groups, torch.float32, keep=keep)
    x, Wu, Wd, ga, be, dout = _block_inputs(images, P, C, F, torch.float32)
    blk.pack_weight(Wd)
    out = blk.forward(x, Wu, ga, be)
    n = R.norm(np64(x), images, groups, "none", "f32", np64(ga), np64(be))["y"]
    within(blk.norm.y, *n, "norm")
    y = R.gated(np64(blk.norm.y), np64(Wu), None, "silu", "f32")["y"]
    within(blk.gated.y, *y, "gated")
    y8, w8 = R.f8_values(*R.f8_pack(blk.gated.y.cpu().numpy())), R.f8_values(*R.f8_pack(Wd.cpu().numpy()))
    want = np64(x) + y8 @ w8.T
    e = (F + 10) * U * (np.abs(y8) @ np.abs(w8).T + np.abs(np64(x)))
    within(out, want, e + U * np.abs(want), "out")
    dx, dgamma, dbeta, dWu, dWd = blk.backward(x, Wu, ga, be, dout)
    d = np64(dout)
    dy = np64(blk.down.dx)
    within(blk.down.dx, d @ w8, (C + 10) * U * (np.abs(d) @ np.abs(w8)), "dy")
    within(dWd, d.T @ y8, (images * P + 10) * U * (np.abs(d).T @ np.abs(y8)), "dW_down")
    gb = R.gated(np64(blk.norm.y), np64(Wu), None, "silu", "f32", dy)
    within(blk.gated.dx, *gb["dx"], "dn")
    within(dWu, *gb["dW"], "dW_up")
    nb = R.norm(np64(x), images, groups, "none", "f32", np64(ga), np64(be), 1e-5, np64(blk.gated.dx), d)
    for got, name in ((dx, "dx"), (dgamma, "dgamma"), (dbeta, "dbeta")):
        within(got, *nb[name], name)


def test_blocks_share_their_rows():
    """Two blocks in a row, the second on the first's buffers, give what blocks of their own give."""
    sizes = (2, 49, 64, 136, 8, torch.bfloat16)
    x, Wu, Wd, ga, be, dout = _block_inputs(*sizes[:4], torch.bfloat16)
    results = []
    for shared in (False, True):
        a = _block(*sizes)
        b = _block(*sizes, share=a if shared else None)
        for blk in (a, b):
            blk.pack_weight(Wd)
        mid = a.forward(x, Wu, ga, be)
        out = b.forward(mid, Wu, ga, be).clone()
        gb = [t.clone() for t in b.backward(mid, Wu, ga, be, dout)]
        ga_ = [t.clone() for t in a.backward(x, Wu, ga, be, gb[0])]
        results.append([out] + gb + ga_)
    assert all(torch.equal(p, q) for p, q in zip(*results))


@pytest.mark.parametrize("keep", [True, False])
def test_block_in_a_graph(keep):
    """Captured once and replayed on new inputs, with eager work between the replays."""
    sizes = (2, 49, 64, 136, 8, torch.bfloat16)
    blk = _block(*sizes, keep=keep)
    x, Wu, Wd, ga, be, dout = _block_inputs(*sizes[:4], torch.bfloat16)

    def step():
        blk.pack_weight(Wd)
        return [blk.forward(x, Wu, ga, be)] + list(blk.backward(x, Wu, ga, be, dout))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(3):
        x.copy_(torch.randn(x.shape, generator=R.gen(20 + i)))
        Wd.mul_(1.25)
        graph.replay()
        got = [t.clone() for t in outs]
        torch.cuda.synchronize()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_calls_on_another_stream_wait_for_nothing_else():
    """Everything a call enqueues, scratch included, is on the stream that it is given."""
    sizes = (2, 49, 64, 136, 8, torch.bfloat16)
    x, Wu, Wd, ga, be, dout = _block_inputs(*sizes[:4], torch.bfloat16)
    blk, ref = _block(*sizes), _block(*sizes)
    ref.pack_weight(Wd)
    want = [ref.forward(x, Wu, ga, be)] + list(ref.backward(x, Wu, ga, be, dout))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    blk.pack_weight(Wd, stream=side)
    got = [blk.forward(x, Wu, ga, be, stream=side)] + list(blk.backward(x, Wu, ga, be, dout, stream=side))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_results_do_not_change_from_run_to_run():
    sizes = (3, 49, 128, 264, 8, torch.bfloat16)
    x, Wu, Wd, ga, be, dout = _block_inputs(*sizes[:4], torch.bfloat16)
    blk = _block(*sizes)
    first = None
    for _ in range(4):
        blk.pack_weight(Wd)
        got = [t.clone() for t in [blk.forward(x, Wu, ga, be)] + list(blk.backward(x, Wu, ga, be, dout))]
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(got, first))


# ---- every tile, split and launch of the products, every walk of group norm ------------------------------------------

# Tiles of 128 and 256 with one and with two workgroups a compute unit, entire sums and parts of them, products in one launch and in two, each with
# tails in every direction
LARGE = [(2000, 130, 3001), (3001, 200, 3500), (3500, 3001, 200), (200, 3001, 3500), (600, 8200, 600), (1000, 4096, 1030), (1568, 2048, 520), (5000, 72, 4100)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", LARGE)
def test_large_f8_linear_of_whole_numbers_is_exact(M, K, N, dtype):
    dt = DT[dtype]
    x, W, dz, addx = (_whole(*s, M + i, m) for i, (s, m) in enumerate([((M, K), 8), ((N, K), 8), ((M, N), 3), ((M, K), 50)]))
    lay = _f8_layer(M, K, N, dtype)
    lay.pack_weight(W.to("cuda", dt))
    z = lay.forward(x.to("cuda", dt))
    assert torch.equal(z.cpu(), (x.double() @ W.double().T).float().to(dt))
    # (the three ways to ask: both products, each alone)
    want_x, want_W = (dz.double() @ W.double() + addx.double()).float().to(dt), (dz.double().T @ x.double()).float().to(dt)
    for need in ((True, True), (True, False), (False, True)):
        lay.dx.fill_(7)
        lay.dW.fill_(7)
        dx, dW, _ = lay.backward(dz.to("cuda", dt), need_dx=need[0], need_dW=need[1], add=addx.to("cuda", dt) if need[0] else None)
        assert dx is None or torch.equal(dx.cpu(), want_x)
        assert dW is None or torch.equal(dW.cpu(), want_W)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,F", [(2000, 130, 1501), (3001, 200, 1750), (2060, 2048, 1026), (600, 4100, 300), (1568, 520, 1024), (5000, 72, 2050)])
def test_large_gated_product(M, K, F, dtype):
    G, dt = _mods()[1], DT[dtype]
    x, W, b, dy = _glu_case(M, K, F, dtype, M + K + F)
    lay = G.Gated(M, K, F, dt, "silu", keep=True)
    xd, Wd, bd, dyd = x.to("cuda", dt), W.to("cuda", dt), b.cuda(), dy.to("cuda", dt)
    y = lay.forward(xd, Wd, bd)
    want = R.gated(*(np64(t) for t in (x, W)), np64(b), "silu", dtype, np64(dy))
    within(y, *want["y"], "y")
    got = [t.clone() for t in lay.backward(xd, Wd, dyd, bd)]
    for t, name in zip(got, ("dx", "dW", "db")):
        within(t, *want[name], name)
    again = G.Gated(M, K, F, dt, "silu", keep=False)      # the projections a second time: the same bits
    assert torch.equal(again.forward(xd, Wd, bd), y)
    assert all(torch.equal(a, b) for a, b in zip(again.backward(xd, Wd, dyd, bd), got))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("images,P,C,G", [(32, 3136, 64, 8), (8, 3136, 256, 32), (40, 49, 2048, 32), (5, 891, 72, 8), (2000, 1, 4096, 1), (1, 40000, 8, 1), (3, 5000, 100, 4)])
def test_group_norm_decides_every_value_next_to_the_border(images, P, C, G, dtype):
    """dy = 1: dbeta is the number of values that passed, which 32 bits hold."""
    N, dt = _mods()[2], DT[dtype]
    for seed in range(3):
        x, ga, be, _ = _norm_case(images, P, C, dtype, 50 + seed)
        lay = N.GroupNorm(images, P, C, G, dt, act="relu")
        xd, gd, bd = x.to("cuda", dt), ga.cuda(), be.cuda()
        lay.forward(xd, gd, bd)
        dbeta = lay.backward(xd, gd, bd, torch.ones_like(xd))[2]
        g4 = xd.double().view(images, P, G, C // G)
        mean = g4.mean((1, 3), keepdim=True)
        r = ((g4 - mean).square().mean((1, 3), keepdim=True) + float(np.float32(1e-5))).rsqrt()
        z = (g4 - mean) * r * gd.double().view(G, -1) + bd.double().view(G, -1)
        assert torch.equal(dbeta.double(), (z > 0).sum((0, 1)).double().view(-1)), seed


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_a_wide_buffer_are_copied_where_they_cannot_be_read_in_place(dtype):
    """Rows 2^21 elements apart, and rows that start off a 16-byte border: the same bits as from rows next to each other."""
    G, dt, M, K, F = _mods()[1], DT[dtype], 40, 64, 48
    x, W, b, dy = _glu_case(M, K, F, dtype, 3)
    results = []
    for gap in (0, (1 << 21) - K, 3):
        lay = G.Gated(M, K, F, dt, "silu", gap=gap)
        xd, dyd = on_device(x, gap, dt), on_device(dy, gap, dt)
        y = lay.forward(xd, W.to("cuda", dt), b.cuda())
        results.append([y.clone()] + [t.clone() for t in lay.backward(xd, W.to("cuda", dt), dyd, b.cuda())])
    for r in results[1:]:
        assert all(torch.equal(p, q) for p, q in zip(r, results[0]))


def test_two_graphs_of_one_block_take_turns():
    """Two captured graphs on one workspace, replayed one after the other, and an eager call between them."""
    sizes = (2, 49, 64, 136, 8, torch.bfloat16)
    blk = _block(*sizes)
    ins = [[t.clone() for t in _block_inputs(*sizes[:4], torch.bfloat16)] for _ in range(2)]
    ins[1][0].mul_(-0.5)

    def step(x, Wu, Wd, ga, be, dout):
        blk.pack_weight(Wd)
        return [t.clone() for t in [blk.forward(x, Wu, ga, be)] + list(blk.backward(x, Wu, ga, be, dout))]

    want = [step(*i) for i in ins]
    graphs, outs = [], []
    for i in ins:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            step(*i)
        torch.cuda.current_stream().wait_stream(side)
        with torch.cuda.graph(graph):
            outs.append(step(*i))
        graphs.append(graph)
    for _ in range(3):
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        step(*ins[0])
        for o, w in zip(outs, want):
            assert all(torch.equal(a, b) for a, b in zip(o, w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["relu", "gelu"])
@pytest.mark.parametrize("images,P,C,G,gap", [(1, 2289, 1472, 1, 8), (1, 676, 2872, 4, 5), (1, 6000, 512, 16, 0), (2, 2000, 300, 300, 3), (3, 700, 130, 65, 0)])
def test_group_norm_of_few_images_in_many_segments(images, P, C, G, gap, act, dtype):
    test_group_norm(images, P, C, G, act, gap, True, dtype)
