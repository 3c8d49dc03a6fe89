"""What is timed of the library's operators for a head behind the backbone: group norm with an activation on channels-last
tensors, the gated feed-forward product, and the matrix product in 8-bit floating point, each with its backward pass.

    norm    xhat = (x - mean) / sqrt(var + eps) over the pixels and channels of a group,  y = f(gamma xhat + beta)
    gated   y = f(x Wg^T + bg) (x Wu^T + bu), W = [Wg; Wu] with 2 F rows
    f8      z = x8 W8^T + b; a row of channels is held in blocks of 128 as e4m3 codes and a power of two 2^e:
                a = max |x| of the block,  e = the least whole number with a <= 448 2^e (not below -116),
                code = e4m3(x 2^-e), ties to even
            backward takes x8 and W8 as they are held:  dx = dz W8,  dW = dz^T x8,  db = column sums of dz

`run` calls the library where `own` is set and computes the same with elementary operations in 32 bits where it is not.
"""
import math

import torch

own = False

EPS = 1e-5
BLOCK = 128


def _norm(images, pixels, C, groups, act="relu", dtype="bf16", train=True, gap=0, name=None):
    c = dict(op="norm", images=images, pixels=pixels, C=C, groups=groups, act=act, dtype=dtype, train=train, gap=gap)
    return dict(c, name=name) if name else c


def _rows(op, M, K, N, dtype="bf16", train=True, bias=False, gap=0, act="silu", name=None):
    """K channels in, N out (gated: N = F, the channels of y).  gap: elements between the end of a row and the next one's start."""
    c = dict(op=op, M=M, K=K, N=N, dtype=dtype, train=train, bias=bias, gap=gap, act=act)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one image's last feature map on its way through a serving program: launches
        _norm(1, 49, 2048, 32, act="silu", train=False, name="norm_49"),
        # a training step of a first-stage block's norm, 32 images
        _norm(32, 3136, 256, 32, name="norm_56"),
        # a small ragged layer in single precision: 5 images of 27 x 33, groups of 9 channels
        _norm(5, 891, 72, 8, act="gelu", dtype="f32", name="norm_27x33"),
        # a training step of a norm over each token's channels, a long batch
        _norm(8192, 1, 4096, 1, act="none", name="norm_tokens"),
        # one token through the gated block of a wide head: latency
        _rows("gated", 1, 2048, 8192, train=False, name="gated_1"),
        # a training step, 32 images' last-stage pixels as tokens
        _rows("gated", 1568, 512, 2048, act="gelu", name="gated_1568"),
        # a small ragged layer in single precision, rows of a wider buffer
        _rows("gated", 777, 136, 72, dtype="f32", bias=True, gap=5, name="gated_777"),
        # a training step of a large block
        _rows("gated", 8192, 4096, 8192, name="gated_8192"),
        # one token through a wide layer whose packed weights are kept: latency
        _rows("f8", 1, 2048, 8192, train=False, bias=True, name="f8_1"),
        # a long prompt
        _rows("f8", 8192, 4096, 8192, train=False, name="f8_8192"),
        # a training step of a last-stage reduction, 32 images' pixels as tokens
        _rows("f8", 1568, 2048, 512, bias=True, name="f8_train_1568"),
        # a training step of a large square layer
        _rows("f8", 8192, 4096, 4096, name="f8_train_8192"),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, spread evenly over its logarithm."""
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def _width(rng, lo, hi):
    """A number of channels: a power of two, an odd multiple of 64 or of 8, or any odd number."""
    k, step = _log(rng, lo, hi), rng.choice([0, 0, 64, 64, 8, 1])
    k = 2 ** round(math.log2(k)) if not step else (k // step | 1) * step
    return max(lo, min(hi, k))


def draw(rng):
    op = rng.choice(["norm", "gated", "f8"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    train, gap = rng.random() < 0.6, rng.choice([0, 0, 0, 8, 5])
    if op == "norm":
        C = _width(rng, 64, 4096)
        most = 2 ** (24 if dtype == "f32" else 25) // C
        if rng.random() < 0.25:
            images, pixels = _log(rng, 1, min(most, 16384)), 1
        else:
            pixels = _log(rng, 4, min(most, 12544))
            images = _log(rng, 1, max(1, min(64, most // pixels)))
        # (64 values a group at least: with two or three dx is what is left of a difference of equal numbers)
        groups = rng.choice([g for g in list(range(1, min(C, 64) + 1)) + [C] if C % g == 0 and pixels * C // g >= 64])
        return _norm(images, pixels, C, groups, rng.choice(["none", "relu", "silu", "gelu"]), dtype, train, gap)
    K, N = _width(rng, 64, 8192), _width(rng, 64, 8192)
    cost = K * N * (6 if op == "gated" else 3) if train else K * N * (2 if op == "gated" else 1)   # a row's multiplies
    most = min(16384, 5 * 10 ** 7 // (K + N), 2 ** (36 if dtype == "f32" else 39) // cost)
    M = _log(rng, 1, most) if train or rng.random() < 0.6 else rng.randrange(1, 33)
    return _rows(op, M, K, N, dtype, train, rng.random() < 0.5, gap, rng.choice(["silu", "gelu"]))


class _State:
    pass


def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _blocks(k):
    return -(-k // BLOCK)


def _inputs(case, seed):
    """The case's tensors, from the seed alone: feature maps with loud channels and means off zero, tokens of which some are all zero
    (padding) and small gradients that are zero for the same tokens, weights of a trained layer's scale."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt, gap = _torch_dtype(case), case["gap"]

    def normal(*size):
        return torch.randn(*size, generator=g, device="cuda")

    def rows(v):
        buf = torch.zeros(v.shape[0], v.shape[1] + gap, dtype=dt, device="cuda")
        buf[:, :v.shape[1]] = v.to(dt)
        return buf[:, :v.shape[1]]

    t = {}
    if case["op"] == "norm":
        M, C = case["images"] * case["pixels"], case["C"]
        t["x"] = rows(normal(M, C) * (0.5 + torch.rand(C, generator=g, device="cuda")) + 0.5 * normal(C))
        t["gamma"], t["beta"] = 1 + 0.3 * normal(C), 0.3 * normal(C)
        if case["train"]:
            t["dy"] = rows(1e-3 * normal(M, C))
        return t
    M, K, N = case["M"], case["K"], case["N"]
    live = (torch.rand(M, 1, generator=g, device="cuda") > 0.03).float()
    live[0] = 1
    loud = 1 + 9 * (torch.rand(K, generator=g, device="cuda") > 0.99).float()
    t["x"] = rows(normal(M, K) * live * loud)
    two = 2 if case["op"] == "gated" else 1
    W = normal(two * N, K) * K ** -0.5
    t["b"] = normal(two * N) * 0.1 if case["bias"] else None
    if case["train"]:
        t["dz"] = rows(1e-3 * normal(M, N) * live)
    if case["op"] == "gated" or case["train"]:
        t["W"] = W.to(dt)
    else:   # the packed weights that a serving program keeps: codes in rows of a multiple of 16 bytes, 2^e as a byte e + 127 in rows of a multiple of 4
        t["w_codes"] = torch.zeros(N, (K + 15) // 16 * 16, dtype=torch.uint8, device="cuda")
        t["w_scales"] = torch.full((N, (_blocks(K) + 3) // 4 * 4), 127, dtype=torch.uint8, device="cuda")
        v = torch.zeros(N, _blocks(K), BLOCK, device="cuda")
        v.view(N, -1)[:, :K] = W
        a = v.abs().amax(2)
        m, e = torch.frexp(a)
        e = (e - 9 + (m > 0.875)).clamp(min=-116)
        q = torch.ldexp(v, -e[:, :, None]).to(torch.float8_e4m3fn).view(torch.uint8)
        t["w_codes"][:, :K] = q.view(N, -1)[:, :K]
        t["w_scales"][:, :_blocks(K)] = (e + 127).to(torch.uint8)
    return t


def prepare(case, seed):
    st = _State()
    st.case, st.dt = case, _torch_dtype(case)
    st.__dict__.update(_inputs(case, seed))
    if own:   # the buffers that the library's caller keeps: outputs, statistics, codes, workspace
        if case["op"] == "norm":
            from paper_2305_11624_amd import norm
            st.layer = norm.GroupNorm(case["images"], case["pixels"], case["C"], case["groups"], st.dt, act=case["act"], eps=EPS,
                                      train=case["train"], gap=case["gap"])
        elif case["op"] == "gated":
            from paper_2305_11624_amd import gated
            st.layer = gated.Gated(case["M"], case["K"], case["N"], st.dt, kind=case["act"], train=case["train"], gap=case["gap"])
        else:
            from paper_2305_11624_amd import quant
            st.layer = quant.F8Linear(case["M"], case["K"], case["N"], st.dt, train=case["train"], gap=case["gap"])
            if not case["train"]:
                st.layer.set_weight(st.w_codes, st.w_scales)
    return st


# ---- the plain forms: elementary operations, 32 bits, rounded once at the end --------------------------------------

def _activation(kind, g):
    """f(g) and f'(g)."""
    if kind == "none":
        return g, torch.ones_like(g)
    if kind == "relu":
        on = (g > 0).float()
        return g * on, on
    if kind == "silu":
        sig = 1.0 / (1.0 + torch.exp(-g))
        return g * sig, sig * (1.0 + g * (1.0 - sig))
    cdf = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_norm(st):
    c, dt = st.case, st.dt
    shape = (c["images"], c["pixels"], c["groups"], c["C"] // c["groups"])
    x = st.x.float().reshape(shape)
    d = x - x.mean((1, 3), keepdim=True)
    r = 1.0 / torch.sqrt((d * d).mean((1, 3), keepdim=True) + EPS)
    xhat = d * r
    gamma, beta = st.gamma.view(shape[2:]), st.beta.view(shape[2:])
    f, df = _activation(c["act"], xhat * gamma + beta)
    out = dict(y=f.reshape(-1, c["C"]).to(dt))
    if c["train"]:
        dz = st.dy.float().reshape(shape) * df
        dxhat = dz * gamma
        dx = r * (dxhat - dxhat.mean((1, 3), keepdim=True) - xhat * (dxhat * xhat).mean((1, 3), keepdim=True))
        out.update(dx=dx.reshape(-1, c["C"]).to(dt), dgamma=(dz * xhat).sum((0, 1)).view(-1), dbeta=dz.sum((0, 1)).view(-1))
    return out


def _plain_gated(st):
    c, dt, F = st.case, st.dt, st.case["N"]
    x, W = st.x.float(), st.W.float()
    h = torch.matmul(x, W.t())
    if st.b is not None:
        h = h + st.b
    g, u = h[:, :F], h[:, F:]
    f, df = _activation(c["act"], g)
    out = dict(y=(f * u).to(dt))
    if c["train"]:
        dy = st.dz.float()
        dh = torch.cat([dy * u * df, dy * f], 1)
        out.update(dx=torch.matmul(dh, W).to(dt), dW=torch.matmul(dh.t(), x).to(dt))
        if st.b is not None:
            out["db"] = dh.sum(0)
    return out


def _f8(x):
    """The values that the codes of the rows of x stand for."""
    M, K = x.shape
    v = torch.zeros(M, _blocks(K) * BLOCK, device=x.device)
    v[:, :K] = x.float()
    v = v.view(M, -1, BLOCK)
    m, e = torch.frexp(v.abs().amax(2))
    e = (e - 9 + (m > 0.875)).clamp(min=-116)[:, :, None]
    return torch.ldexp(torch.ldexp(v, -e).to(torch.float8_e4m3fn).float(), e).view(M, -1)[:, :K]


def _plain_f8(st):
    dt, K = st.dt, st.case["K"]
    x = _f8(st.x)
    if st.case["train"]:
        w = _f8(st.W)
    else:
        two = torch.ldexp(torch.ones(1, device=x.device), st.w_scales[:, :_blocks(K)].int() - 127)
        w = st.w_codes[:, :K].view(torch.float8_e4m3fn).float() * torch.repeat_interleave(two, BLOCK, 1)[:, :K]
    z = torch.matmul(x, w.t())
    if st.b is not None:
        z = z + st.b
    out = dict(z=z.to(dt))
    if st.case["train"]:
        dz = st.dz.float()
        out.update(dx=torch.matmul(dz, w).to(dt), dW=torch.matmul(dz.t(), x).to(dt))
        if st.b is not None:
            out["db"] = dz.sum(0)
    return out


def run(state):
    op, train = state.case["op"], state.case["train"]
    if not own:
        return (_plain_norm if op == "norm" else _plain_gated if op == "gated" else _plain_f8)(state)
    layer = state.layer
    if op == "norm":
        y = layer.forward(state.x, state.gamma, state.beta)
        if not train:
            return dict(y=y)
        dx, dgamma, dbeta = layer.backward(state.x, state.gamma, state.beta, state.dy)
        return dict(y=y, dx=dx, dgamma=dgamma, dbeta=dbeta)
    if op == "gated":
        out = dict(y=layer.forward(state.x, state.W, state.b))
        if train:
            out["dx"], out["dW"], db = layer.backward(state.x, state.W, state.dz, b=state.b)
    else:
        if train:
            layer.pack_weight(state.W)
        out = dict(z=layer.forward(state.x, state.b))
        if train:
            out["dx"], out["dW"], db = layer.backward(state.dz, bias=state.b is not None)
    if train and db is not None:
        out["db"] = db
    return out


def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "norm":   # x in, y out; x and dy in, dx out; gamma, beta, their gradients and the statistics
        n, C = case["images"] * case["pixels"] * case["C"], case["C"]
        stats = 8 * case["images"] * case["groups"]
        if case["train"]:
            return {"bytes": float(5 * n * e + 24 * C + 2 * stats), "flops": 40.0 * n}
        return {"bytes": float(2 * n * e + 8 * C), "flops": 16.0 * n}
    M, K, N = case["M"], case["K"], case["N"]
    if case["op"] == "gated":   # x, W in, y out; x, W, dy in, dx, dW out (what is kept of h comes on top)
        if case["train"]:
            return {"bytes": float(e * (3 * M * K + 6 * N * K + 2 * M * N)), "flops": 12.0 * M * N * K}
        return {"bytes": float(e * (M * K + 2 * N * K + M * N)), "flops": 4.0 * M * N * K}
    held = K + _blocks(K)
    if case["train"]:   # x, W, dz in, z, dx, dW out; the codes of x and W are written once and read in backward
        return {"bytes": float(2 * e * (M * K + N * K + M * N) + 2 * held * (M + N)), "flops": 6.0 * M * N * K}
    return {"bytes": float(M * K * e + N * held + M * N * e), "flops": 2.0 * M * N * K}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------
# Gradients come from automatic differentiation of the forward definition; the codes are whole numbers of steps.

def _f64(kind, g):
    if kind == "none":
        return g
    if kind == "relu":
        return torch.clamp(g, min=0)
    if kind == "silu":
        return g * torch.sigmoid(g)
    return g * 0.5 * torch.special.erfc(-g / math.sqrt(2.0))


def _held64(x):
    """The values that rows are held as: e from a logarithm, then the nearest of the e4m3 numbers by whole steps."""
    x = x.double()
    M, K = x.shape
    at = torch.arange(K, device=x.device) // BLOCK
    a = torch.stack([x[:, i:i + BLOCK].abs().max(dim=1)[0] for i in range(0, K, BLOCK)], 1)
    e = torch.ceil(torch.log2(torch.clamp(a, min=2.0 ** -140) / 448.0)).clamp(min=-116.0)
    v = x * torch.exp2(-e)[:, at]
    step = torch.exp2(torch.floor(torch.log2(torch.clamp(v.abs(), min=2.0 ** -6))) - 3.0)
    return torch.round(v / step) * step * torch.exp2(e)[:, at]


def exact(case, seed):
    t, train = _inputs(case, seed), case["train"]
    if case["op"] == "norm":
        n, p, C, G = (case[k] for k in ("images", "pixels", "C", "groups"))
        x = t["x"].double().requires_grad_(train)
        gamma, beta = (t[k].double().requires_grad_(train) for k in ("gamma", "beta"))
        per = x.view(n, p, G, C // G).transpose(1, 2).reshape(n, G, -1)
        var, mean = torch.var_mean(per, dim=2, unbiased=False)
        spread = lambda s: s.repeat_interleave(C // G, 1).repeat_interleave(p, 0)
        xhat = (x - spread(mean)) / torch.sqrt(spread(var) + EPS)
        y = _f64(case["act"], xhat * gamma + beta)
        if not train:
            return dict(y=y)
        dx, dgamma, dbeta = torch.autograd.grad(y, (x, gamma, beta), t["dy"].double())
        return dict(y=y.detach(), dx=dx, dgamma=dgamma, dbeta=dbeta)
    if case["op"] == "gated":
        x, W = (t[k].double().requires_grad_(train) for k in ("x", "W"))
        b = None if t["b"] is None else t["b"].double().requires_grad_(train)
        F = case["N"]
        g, u = x @ W[:F].T, x @ W[F:].T
        if b is not None:
            g, u = g + b[:F], u + b[F:]
        y = _f64(case["act"], g) * u
        if not train:
            return dict(y=y)
        leaves = dict(dx=x, dW=W) if b is None else dict(dx=x, dW=W, db=b)
        return dict(y=y.detach(), **dict(zip(leaves, torch.autograd.grad(y, tuple(leaves.values()), t["dz"].double()))))
    x, K = _held64(t["x"]), case["K"]
    if train:
        w = _held64(t["W"])
    else:
        w = t["w_codes"][:, :K].view(torch.float8_e4m3fn).double()
        w = w * torch.exp2(t["w_scales"].double() - 127.0)[:, torch.arange(K, device=w.device) // BLOCK]
    z = x @ w.T.contiguous()
    if t["b"] is not None:
        z += t["b"].double()
    if not train:
        return dict(z=z)
    dz = t["dz"].double()
    out = dict(z=z, dx=dz @ w, dW=dz.T.contiguous() @ x)
    if t["b"] is not None:
        out["db"] = dz.sum(dim=0)
    return out
