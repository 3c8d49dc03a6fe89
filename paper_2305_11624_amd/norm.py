"""Group norm with an activation on channels-last tensors, for a PyTorch program.

The object holds the outputs, statistics and workspace of one layer, allocated once; its calls enqueue on the current stream (or the one they are
given) and allocate nothing.  What they return are the object's own buffers, overwritten by the next call.  Types, sizes and strides of the
arguments are checked before anything is launched (ValueError)."""
from typing import Optional

import torch

from . import binding as B
from .quant import _dtype, _rows

_ACTS = {"none": B.NORM_NONE, "relu": B.NORM_RELU, "silu": B.NORM_SILU, "gelu": B.NORM_GELU}


def workspace_bytes(images: int, pixels: int, C: int, groups: int, dtype=torch.bfloat16, train: bool = True, gap: int = 0) -> int:
    """What `GroupNorm` of these sizes needs as its `ws`."""
    d = B.make_norm_desc(images, pixels, C, groups, _dtype(dtype), C + gap, C + gap)
    return max(B.convbn_norm_workspace_bytes(d, p) for p in ((B.PASS_FWD, B.PASS_BWD) if train else (B.PASS_FWD,)))


class GroupNorm:
    """y = f(gamma (x - mean) / sqrt(var + eps) + beta), f = act ("none", "relu", "silu", "gelu"), with mean and variance over the pixels and
    channels of each of an image's `groups` groups.  x: [images * pixels, C] rows, the channels-last tensor as it lies in memory.  (pixels = 1,
    groups = 1: a norm over each token's channels.)

    train: the statistics are kept for `backward`, which reads x again.  gap: x, dx, y and dy are rows of buffers with `gap` elements
    between the rows.  y, dx: rows that the layer writes, ws: bytes that it works in (`workspace_bytes`), where several layers share them."""

    def __init__(self, images: int, pixels: int, C: int, groups: int, dtype=torch.bfloat16, act: str = "none", eps: float = 1e-5,
                 train: bool = True, gap: int = 0, device="cuda", y: Optional[torch.Tensor] = None, dx: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None):
        if act not in _ACTS:
            raise ValueError(f"act: {act!r}, expected one of {sorted(_ACTS)}")
        self.rows, self.C, self.dtype, self.ld = images * pixels, C, dtype, C + gap
        self.desc, self._add_desc = (B.make_norm_desc(images, pixels, C, groups, _dtype(dtype), self.ld, self.ld, _ACTS[act], eps)
                                     for _ in range(2))   # (the second with an addend)
        self.y = _rows(y, self.rows, C, self.ld, dtype, device, "y")
        self.dx = _rows(dx, self.rows, C, self.ld, dtype, device, "dx") if train else None
        self.stats = torch.empty(images * groups * 4, dtype=torch.float32, device=device) if train else None
        self.dgamma, self.dbeta = (torch.empty(C, dtype=torch.float32, device=device) if train else None for _ in range(2))
        need = workspace_bytes(images, pixels, C, groups, dtype, train, gap)
        if ws is not None and ws.nbytes < need:
            raise ValueError(f"ws: {ws.nbytes} bytes, {need} needed")
        self.ws = ws if ws is not None else torch.empty(need, dtype=torch.uint8, device=device) if need else None

    def forward(self, x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None, stream=None):
        """gamma, beta: float32 [C]; None = ones, zeros."""
        if x is None:
            raise ValueError("x: expected rows")
        B.convbn_norm_fwd(self.desc, x, gamma, beta, self.y, self.stats, self.ws, stream)
        return self.y

    def backward(self, x: torch.Tensor, gamma: Optional[torch.Tensor], beta: Optional[torch.Tensor], dy: torch.Tensor,
                 need_dx: bool = True, need_params: bool = True, add: Optional[torch.Tensor] = None, stream=None):
        """(dx (+ add), dgamma, dbeta) for the x, gamma and beta of the last forward; None for what is not asked for."""
        if self.stats is None:
            raise RuntimeError("this layer keeps no statistics (train=False)")
        if x is None or dy is None:
            raise ValueError("x, dy: expected rows")
        d = self.desc
        if add is not None:
            if (add.dtype is not self.dtype or add.shape != (self.rows, self.C) or self.rows > 1 and add.stride(0) != self.ld
                    or self.rows and self.C > 1 and add.stride(1) != 1 or add.device != self.y.device):
                raise ValueError(f"add: expected {self.dtype} [{self.rows}, {self.C}] with rows {self.ld} elements apart on {self.y.device}")
            d = self._add_desc
            d.act, d.add_in = B.ACT_ADD_IN, add.data_ptr()
        dx, dgamma, dbeta = self.dx if need_dx else None, self.dgamma if need_params else None, self.dbeta if need_params else None
        B.convbn_norm_bwd(d, x, gamma, beta, self.stats, dy, dx, dgamma, dbeta, self.ws, stream)
        return dx, dgamma, dbeta

    def saved_bytes(self) -> int:
        """The statistics: what backward needs of the forward pass beside x."""
        return 0 if self.stats is None else self.stats.nbytes
