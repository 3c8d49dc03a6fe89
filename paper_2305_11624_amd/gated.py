"""The gated feed-forward product in bf16 or fp32, and the block that it makes up with a norm in front and a product in 8-bit floating point behind.

Each object holds the outputs and the workspace of one layer, allocated once; its calls enqueue on the current stream (or the one they are given)
and allocate nothing, but for the first `pack_weight` of the block's last product.  What they return are the object's own buffers, overwritten by
the next call.  Types, sizes and strides of the arguments are checked before anything is launched (ValueError)."""
from typing import Optional

import torch

from . import binding as B
from . import norm as _norm
from . import quant as Q
from .quant import _GATES, _dtype, _rows


def workspace_bytes(M: int, C: int, F: int, dtype=torch.bfloat16, train: bool = True, gap: int = 0, keep: bool = False) -> int:
    """What `Gated` of these sizes needs as its `ws`; keep: one that keeps h, which needs less."""
    d = B.make_qdesc(M, C, F, _dtype(dtype), C + gap, F + gap, act=B.ACT_H_KEPT if keep else 0)
    return max(B.convbn_glu_workspace_bytes(d, p) for p in ((B.PASS_FWD, B.PASS_BWD) if train else (B.PASS_FWD,)))


class Gated:
    """y = f(x Wg^T + bg) (x Wu^T + bu) on M rows of C channels, F out: both projections, f = "silu" or "gelu" and the product in one call.
    W = [Wg; Wu] is [2 F, C] (g's rows first), b = [bg; bu] float32 [2 F] or None.

    train: there are buffers for `backward`, which reads x and W again.  keep: h = [g | u] is kept for it, in float32; without, it multiplies x and W
    once more, with the same result, and 2 F numbers a row need not be kept.  gap: x, dx, y and dy are rows of buffers with `gap` elements between the rows.  y, dx: rows that the
    layer writes, ws: bytes that it works in (`workspace_bytes`), where several layers share them."""

    def __init__(self, M: int, C: int, F: int, dtype=torch.bfloat16, kind: str = "silu", train: bool = True, keep: bool = True, gap: int = 0,
                 device="cuda", y: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
        if kind not in _GATES:
            raise ValueError(f"kind: {kind!r}, expected one of {sorted(_GATES)}")
        self.M, self.C, self.F, self.dtype, self.train = M, C, F, dtype, train
        self.ldx, self.ldy = C + gap, F + gap
        self._act = B.ACT_H_KEPT if train and keep else 0
        self.desc, self._add_desc = (B.make_qdesc(M, C, F, _dtype(dtype), self.ldx, self.ldy, self._act, _GATES[kind]) for _ in range(2))
        self.y = _rows(y, M, F, self.ldy, dtype, device, "y")
        self.h = torch.empty(M, 2 * F, dtype=torch.float32, device=device) if train and keep else None
        self.dx = _rows(dx, M, C, self.ldx, dtype, device, "dx") if train else None
        self.dW = torch.empty(2 * F, C, dtype=dtype, device=device) if train else None
        self.db = torch.empty(2 * F, dtype=torch.float32, device=device) if train else None
        need = workspace_bytes(M, C, F, dtype, train, gap, keep)
        if ws is not None and ws.nbytes < need:
            raise ValueError(f"ws: {ws.nbytes} bytes, {need} needed")
        self.ws = ws if ws is not None else torch.empty(need, dtype=torch.uint8, device=device) if need else None

    def forward(self, x: torch.Tensor, W: torch.Tensor, b: Optional[torch.Tensor] = None, stream=None):
        if x is None or W is None:
            raise ValueError("x, W: expected rows and a weight")
        B.convbn_glu_fwd(self.desc, x, W, b, self.y, self.h, self.ws, stream)
        return self.y

    def backward(self, x: torch.Tensor, W: torch.Tensor, dy: torch.Tensor, b: Optional[torch.Tensor] = None, need_dx: bool = True,
                 need_dW: bool = True, add: Optional[torch.Tensor] = None, stream=None):
        """(dx (+ add), dW, db) for the x, W and b of the last forward; None for what is not asked for, and for db without b."""
        if not self.train:
            raise RuntimeError("this layer has no buffers for a backward pass (train=False)")
        if x is None or W is None or dy is None:
            raise ValueError("x, W, dy: expected rows and a weight")
        d = self.desc
        if add is not None:
            if (add.dtype is not self.dtype or add.shape != (self.M, self.C) or self.M > 1 and add.stride(0) != self.ldx
                    or self.M and self.C > 1 and add.stride(1) != 1 or add.device != self.y.device):
                raise ValueError(f"add: expected {self.dtype} [{self.M}, {self.C}] with rows {self.ldx} elements apart on {self.y.device}")
            d = self._add_desc
            d.act, d.add_in = self._act | B.ACT_ADD_IN, add.data_ptr()
        dx, dW, db = self.dx if need_dx else None, self.dW if need_dW else None, self.db if b is not None else None
        B.convbn_glu_bwd(d, x, W, b, self.h, dy, dx, dW, db, self.ws, stream)
        return dx, dW, db

    def saved_bytes(self) -> int:
        """h: what backward needs of the forward pass beside x and W."""
        return 0 if self.h is None else self.h.nbytes


class NormGatedBlock:
    """out = x + down(gated(norm(x))): a residual block on channels-last rows, `images` images of `pixels` pixels (tokens: pixels = 1, groups = 1) of C
    channels with F hidden ones.  The norm has `groups` groups, the gated product runs in dtype, the product back to C channels in 8-bit
    floating point.  Backward needs x, the norm's output and statistics, the codes of y and, with keep, h.

    share: a block of the same sizes whose y, gradients of rows and workspace this one uses too, as the blocks of a stack do."""

    def __init__(self, images: int, pixels: int, C: int, F: int, groups: int = 1, dtype=torch.bfloat16, kind: str = "silu", eps: float = 1e-5,
                 train: bool = True, keep: bool = True, device="cuda", share: Optional["NormGatedBlock"] = None):
        M = images * pixels
        if share is None:
            need = max(_norm.workspace_bytes(images, pixels, C, groups, dtype, train), workspace_bytes(M, C, F, dtype, train, keep=keep),
                       Q.f8_linear_workspace_bytes(M, F, C, dtype, train))
            ws = torch.empty(need, dtype=torch.uint8, device=device) if need else None
            y = dy = dn = dx = None
        else:
            if train and not share.gated.train:
                raise ValueError("share: a block that is not trained has no gradients to share")
            ws, y, dy, dn, dx = share.gated.ws, share.gated.y, share.down.dx, share.gated.dx, share.norm.dx
        self.norm = _norm.GroupNorm(images, pixels, C, groups, dtype, eps=eps, train=train, device=device, dx=dx, ws=ws)
        self.gated = Gated(M, C, F, dtype, kind, train, keep, device=device, y=y, dx=dn, ws=ws)
        self.down = Q.F8Linear(M, F, C, dtype, train, device=device, dx=dy, ws=ws)

    def pack_weight(self, W_down: torch.Tensor, stream=None):
        """W_down [C, F]: once for serving, every step in training."""
        self.down.pack_weight(W_down, stream)

    def forward(self, x: torch.Tensor, W_up: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, stream=None):
        """W_up [2 F, C]: g's rows before u's."""
        y = self.gated.forward(self.norm.forward(x, gamma, beta, stream), W_up, stream=stream)
        return self.down.forward(y, add=x, stream=stream)

    def backward(self, x: torch.Tensor, W_up: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], dout: torch.Tensor, stream=None):
        """(dx, dgamma, dbeta, dW_up, dW_down) for the x, W_up, gamma and beta of the last forward."""
        dy, dW_down, _ = self.down.backward(dout, stream=stream)
        dn, dW_up, _ = self.gated.backward(self.norm.y, W_up, dy, stream=stream)
        dx, dgamma, dbeta = self.norm.backward(x, gamma, beta, dn, add=dout, stream=stream)
        return dx, dgamma, dbeta, dW_up, dW_down

    def saved_bytes(self) -> int:
        """What backward needs of the forward pass beside x."""
        return self.norm.y.nbytes + self.norm.saved_bytes() + self.gated.saved_bytes() + self.down.saved_bytes()
