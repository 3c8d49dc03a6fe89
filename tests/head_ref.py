"""Plain implementations, in 64 bits on the CPU, of the operators for a head: rows in 8-bit floating point, the gated product, group norm."""
import math

import numpy as np
import torch

U, H = 2.0 ** -24, 2.0 ** -8          # half a step of fp32 and of bf16, relative
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def half(dtype):
    return H if dtype == "bf16" else U


def gen(seed):
    return torch.Generator().manual_seed(seed)


def on_device(x, gap, dt):
    """x on the device, as rows of a buffer with `gap` poisoned elements behind each."""
    buf = torch.full((x.shape[0], x.shape[1] + gap), float("nan"), dtype=dt, device="cuda")
    buf[:, :x.shape[1]] = x.to("cuda", dt)
    return buf[:, :x.shape[1]]


def np64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def within(got, want, allowed, name=""):
    """Element by element; NaN nowhere."""
    got, want, allowed = np64(got) if isinstance(got, torch.Tensor) else got, np.asarray(want), np.asarray(allowed)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    over = np.abs(got - want) - allowed
    assert np.isfinite(got).all(), name
    if over.size and over.max() > 0:
        at = np.unravel_index(over.argmax(), over.shape)
        raise AssertionError("%s at %s: %.9g, expected %.9g, allowed %.3g" % (name, at, got[at], want[at], np.broadcast_to(allowed, want.shape)[at]))


# ---- 8-bit floating point ------------------------------------------------------------------------------------------

def e4m3_values():
    """What the codes 0 .. 255 stand for (127 and 255: NaN)."""
    v = np.zeros(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        v[c] = (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)) * (-1 if c & 128 else 1)
    v[[127, 255]] = np.nan
    return v


_POSITIVE = e4m3_values()[:127]


def to_e4m3(v):
    """Codes of the nearest numbers, ties to the even code; v at most 448 in size."""
    a = np.abs(v)
    hi = np.clip(np.searchsorted(_POSITIVE, a), 1, 126)
    up, down = _POSITIVE[hi] - a, a - _POSITIVE[hi - 1]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def f8_pack(x):
    """(codes [M, K], scale bytes [M, blocks]) of fp32 rows, by the definition."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    M, K = x.shape
    codes, scales = np.zeros((M, K), np.uint8), np.zeros((M, -(-K // 128)), np.uint8)
    for b in range(scales.shape[1]):
        blk = x[:, b * 128:(b + 1) * 128]
        for m in range(M):
            v = blk[m]
            if not np.isfinite(v).all():
                codes[m, b * 128:(b + 1) * 128], scales[m, b] = 127, 127
                continue
            a = np.abs(v).max()
            e = -116
            while a > math.ldexp(448.0, e):
                e += 1
            q = v * 2.0 ** -e
            if e == 120:
                q = np.clip(q, -240, 240)
            codes[m, b * 128:(b + 1) * 128], scales[m, b] = to_e4m3(q), e + 127
    return codes, scales


def f8_values(codes, scales):
    K = codes.shape[1]
    return e4m3_values()[codes] * np.exp2(scales.astype(np.float64) - 127)[:, np.arange(K) // 128]


# ---- activations ---------------------------------------------------------------------------------------------------

def act(kind, g):
    """f, f' and a bound of |f''| everywhere."""
    if kind == "none":
        return g, np.ones_like(g), 0.0
    if kind == "relu":
        return np.maximum(g, 0), (g > 0).astype(np.float64), 0.0
    if kind == "silu":
        p = 1 / (1 + np.exp(-g))
        return g * p, p * (1 + g * (1 - p)), 0.5
    p = 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-g / math.sqrt(2)) if g.size else g
    d = np.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    return g * p, p + g * d, 0.8


def act_error(kind, dtype, g):
    """How far f (relative) and f' (absolute) may be off where they are computed: the hardware's exponential and reciprocal, the fitted tail."""
    if kind in ("none", "relu"):
        return 0.0, 0.0
    if kind == "silu":
        r = (8 if dtype == "f32" else 2 * (2 + np.abs(g)) + 4) * U
    else:
        r = (24 + 1.5 * g * g) * U
    return r, r * (1.2 + np.abs(g)) + 8 * U


# ---- gated product -------------------------------------------------------------------------------------------------

def gated(x, W, b, kind, dtype, dy=None, add=None):
    """Results and how far each may be off: {name: (value, allowed)}.  Sums of R terms t: (R + 8) U sum |t|; each rounding half a step."""
    M, K = x.shape
    F, hs = W.shape[0] // 2, half(dtype)
    bb = np.zeros(2 * F) if b is None else b
    h = x @ W.T + bb
    dh_ = (K + 10) * U * (np.abs(x) @ np.abs(W).T + np.abs(bb))
    g, u, dg, du = h[:, :F], h[:, F:], dh_[:, :F], dh_[:, F:]
    f, df, ddf = act(kind, g)
    rf, rdf = act_error(kind, dtype, g)
    slope = np.abs(df) + ddf * dg      # (on the way from g to what stands for it)
    ef = slope * dg + rf * (np.abs(f) + slope * dg)
    y = f * u
    ey = ef * (np.abs(u) + du) + np.abs(f) * du + 2 * U * np.abs(y)
    out = dict(y=(y, ey + hs * (np.abs(y) + ey)))
    if dy is None:
        return out
    edf = ddf * dg + rdf
    gu = np.concatenate([dy * u * df, dy * f], 1)
    e = np.concatenate([np.abs(dy) * ((np.abs(u) + du) * edf + np.abs(df) * du), np.abs(dy) * ef], 1) + 3 * U * np.abs(gu)
    eb = (M + 10) * U * (np.abs(gu) + e).sum(0) + e.sum(0)
    out["db"] = (gu.sum(0), eb)
    if dtype == "bf16":
        e = e + H * (np.abs(gu) + e)
    dx = gu @ W + (0 if add is None else add)
    ex = e @ np.abs(W) + (2 * F + 10) * U * ((np.abs(gu) + e) @ np.abs(W) + (0 if add is None else np.abs(add)))
    dW = gu.T @ x
    ew = e.T @ np.abs(x) + (M + 10) * U * ((np.abs(gu) + e).T @ np.abs(x))
    out["dx"] = (dx, ex + hs * (np.abs(dx) + ex))
    out["dW"] = (dW, ew + hs * (np.abs(dW) + ew))
    return out


# ---- group norm ----------------------------------------------------------------------------------------------------

def norm(x, images, groups, kind, dtype, gamma=None, beta=None, eps=1e-5, dy=None, add=None):
    """Results and how far each may be off.  No chain of additions is longer than a 64th of a group's values, and some: k U of the sum of the sizes."""
    C, hs = x.shape[1], half(dtype)
    P, cg = x.shape[0] // images, C // groups
    n = P * cg
    k = n / 64 + 40
    g4 = x.reshape(images, P, groups, cg)
    ax = lambda v: v.mean(axis=(1, 3), keepdims=True)
    mean = ax(g4)
    emean = k * U * ax(np.abs(g4))
    d = g4 - mean
    var = ax(d * d)
    evar = (k + 4) * U * var + emean ** 2      # (a mean that is off by e: the sum of (d - e)^2 is that of d^2 and e^2, the d add up to nothing)
    r = 1 / np.sqrt(var + eps)
    er = 0.5 * r ** 3 * evar * 1.5 + 4 * U * r      # (evar far below var + eps: checked)
    assert (evar < 0.1 * (var + eps)).all()
    xhat = d * r
    ed = emean + U * np.abs(d) + 2 * U * np.abs(g4)
    exh = ed * (r + er) + np.abs(d) * er + 2 * U * np.abs(xhat)
    ga = np.ones(C) if gamma is None else gamma
    be = np.zeros(C) if beta is None else beta
    gr, br = ga.reshape(1, 1, groups, cg), be.reshape(1, 1, groups, cg)
    z = xhat * gr + br
    ez = exh * np.abs(gr) + 3 * U * (np.abs(xhat * gr) + np.abs(br))
    f, df, ddf = act(kind, z)
    rf, rdf = act_error(kind, dtype, z)
    slope = np.maximum(np.abs(df) + ddf * ez, 1.0 if kind == "relu" else 0.0)
    ef = slope * ez + rf * (np.abs(f) + slope * ez)
    two = lambda v: np.broadcast_to(v, g4.shape).reshape(x.shape)
    out = dict(y=(two(f), two(ef + hs * (np.abs(f) + ef))), mean=(mean.reshape(-1), emean.reshape(-1)), rstd=(r.reshape(-1), er.reshape(-1)))
    if dy is None:
        return out
    q = dy.reshape(g4.shape)
    dz = q * df
    edf = ddf * ez + rdf + (np.abs(z) <= ez if kind == "relu" else 0)      # (a value next to the border may fall on either side)
    edz = np.abs(q) * edf + 2 * U * np.abs(dz)
    sx, se = dz * xhat, edz * (np.abs(xhat) + exh) + np.abs(dz) * exh
    kk = (images * P) / 64 + images + 40
    out["dbeta"] = (dz.sum(axis=(0, 1)).reshape(-1), (edz.sum(axis=(0, 1)) + kk * U * (np.abs(dz) + edz).sum(axis=(0, 1))).reshape(-1))
    out["dgamma"] = (sx.sum(axis=(0, 1)).reshape(-1), (se.sum(axis=(0, 1)) + kk * U * (np.abs(sx) + se).sum(axis=(0, 1))).reshape(-1))
    dxh, edxh = dz * gr, edz * np.abs(gr) + U * np.abs(dz * gr)
    m1, em1 = ax(dxh), ax(edxh) + (k + P / 64) * U * ax(np.abs(dxh) + edxh)
    m2 = ax(dxh * xhat)
    e2 = edxh * (np.abs(xhat) + exh) + np.abs(dxh) * exh
    em2 = ax(e2) + (k + P / 64) * U * ax(np.abs(dxh * xhat) + e2)
    inner = dxh - m1 - xhat * m2
    einner = edxh + em1 + np.abs(xhat) * em2 + exh * (np.abs(m2) + em2) + 4 * U * (np.abs(dxh) + np.abs(m1) + np.abs(xhat * m2))
    dx = r * inner
    edx = (r + er) * einner + er * np.abs(inner)
    dx, edx = two(dx), two(edx)
    if add is not None:
        edx = edx + 2 * U * (np.abs(dx) + np.abs(add))
        dx = dx + add
    out["dx"] = (dx, edx + hs * (np.abs(dx) + edx))
    return out
