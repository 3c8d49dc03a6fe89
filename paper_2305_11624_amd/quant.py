"""The 8-bit rows for a PyTorch program: an activation kept in 8 bits, a Linear block on integer products that keeps its input
that way, the gate between two of them, and the gated block that they make up; the checkpoint and the Linear block in 8-bit floating point too.

Each object holds the codes, scales, outputs and workspace of one layer, allocated once; its calls enqueue on the current
stream (or the one they are given) and allocate nothing, but for the first `pack_weight` and the first `unpack` without `out`, whose
buffers belong to the stream of that call.  What they return are the object's own buffers, overwritten by the
next call.

What stays between forward and backward are codes and scales: `saved_bytes()`.  The full-width tensors that an object writes (z, dx, y,
dh, what a checkpoint reads back to) and its workspace are scratch, but allocated memory all the same: layers that run one after
the other are given the same ones (z=, dx=, y=, dh=, out=, ws=; `GatedBlock(share=)`), and each further layer then adds codes, scales, its
packed weight and dW alone.  Types, sizes and strides of the arguments are checked before anything is launched (ValueError).
"""
import contextlib
from typing import Optional

import torch

from . import binding as B

_DTYPES = {torch.bfloat16: B.BF16, torch.float32: B.F32}
_GATES = {"silu": B.GATE_SILU, "gelu": B.GATE_GELU}


def _dtype(dt):
    if dt not in _DTYPES:
        raise TypeError(f"{dt}: bfloat16 or float32")
    return _DTYPES[dt]


def _vector(t: Optional[torch.Tensor], n: int, name: str):
    if t is not None and (t.dtype is not torch.float32 or t.numel() != n):
        raise ValueError(f"{name}: expected float32 [{n}], got {t.dtype} {list(t.shape)}")
    return t


def _bytes(t: torch.Tensor, rows: int, width: int, name: str):
    if t.element_size() != 1 or t.dim() != 2 or t.shape[0] != rows or t.shape[1] != width:
        raise ValueError(f"{name}: expected bytes [{rows}, {width}], got {t.dtype} {list(t.shape)}")
    return t


def _codes(t: torch.Tensor, rows: int, K: int, name: str):
    return _bytes(t, rows, B.convbn_qrow_bytes(K), name)


def _rows(given: Optional[torch.Tensor], M, width, ld, dt, device, name: str):
    """Rows for an output: the caller's, or new ones."""
    if given is None:
        return torch.empty(M, ld, dtype=dt, device=device)[:, :width]
    if (given.dtype is not dt or given.shape != (M, width) or M > 1 and given.stride(0) != ld or M and width > 1 and given.stride(1) != 1
            or given.device.type != torch.device(device).type):
        raise ValueError(f"{name}: expected {dt} [{M}, {width}] with rows {ld} elements apart on {device}")
    return given


def _allocating_for(stream):
    """A context whose allocations come from the pool of the stream that a call works on."""
    if stream is None:
        return contextlib.nullcontext()
    return torch.cuda.stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(int(stream)))


def new_codes(rows: int, K: int, device="cuda"):
    """Buffers for `rows` packed rows of K channels: (codes, scales)."""
    return (torch.empty(rows, B.convbn_qrow_bytes(K), dtype=torch.int8, device=device),
            torch.empty(rows, dtype=torch.float32, device=device))


def new_f8_codes(rows: int, K: int, device="cuda"):
    """Buffers for `rows` rows of K channels packed in 8-bit floating point: (codes, scales), a byte e + 127 for each block of 128 channels."""
    return (torch.empty(rows, B.convbn_qrow_bytes(K), dtype=torch.uint8, device=device),
            torch.empty(rows, B.convbn_fscale_bytes(K), dtype=torch.uint8, device=device))


class _IntRows:
    """Codes from -127 to 127, a scale for each row: the calls that work on them."""
    new = staticmethod(lambda rows, K, device: new_codes(rows, K, device))
    pack = staticmethod(lambda *a: B.convbn_qpack(*a))
    unpack = staticmethod(lambda *a: B.convbn_qunpack(*a))
    fwd = staticmethod(lambda *a: B.convbn_qlinear_fwd(*a))
    bwd = staticmethod(lambda *a: B.convbn_qlinear_bwd(*a))
    workspace_bytes = staticmethod(lambda desc, pass_: B.convbn_qlinear_workspace_bytes(desc, pass_))
    scales = staticmethod(lambda t, rows, K, name: _vector(t, rows, name))
    scale_bytes = staticmethod(lambda K: 4)   # of a row


class _F8Rows:
    """e4m3 codes, a power of two for each block of 128 channels of a row."""
    new = staticmethod(lambda rows, K, device: new_f8_codes(rows, K, device))
    pack = staticmethod(lambda *a: B.convbn_fpack(*a))
    unpack = staticmethod(lambda *a: B.convbn_funpack(*a))
    fwd = staticmethod(lambda *a: B.convbn_flinear_fwd(*a))
    bwd = staticmethod(lambda *a: B.convbn_flinear_bwd(*a))
    workspace_bytes = staticmethod(lambda desc, pass_: B.convbn_flinear_workspace_bytes(desc, pass_))
    scales = staticmethod(lambda t, rows, K, name: _bytes(t, rows, B.convbn_fscale_bytes(K), name))
    scale_bytes = staticmethod(lambda K: B.convbn_fscale_bytes(K))


class Checkpoint:
    """[M, K] rows kept in 8 bits between a block's forward and its backward (a channels-last activation is [pixels,
    channels]): 1 byte a value and 4 a row in place of 2 or 4 a value.

    out: dense rows that `unpack` writes; without it (and without `unpack(out)`) the checkpoint allocates and holds some of its own, so several
    checkpoints are better given one buffer."""

    _form = _IntRows

    def __init__(self, M: int, K: int, dtype=torch.bfloat16, device="cuda", out: Optional[torch.Tensor] = None):
        self.M, self.K, self.dtype = M, K, dtype
        self.desc = B.make_qdesc(M, K, dtype=_dtype(dtype))
        self.codes, self.scales = self._form.new(M, K, device)
        self.out = None if out is None else _rows(out, M, K, K, dtype, device, "out")

    def pack(self, x: torch.Tensor, stream=None):
        """The rows of x may be strided."""
        self.desc.ldx = x.stride(0) if self.M > 1 else self.K
        self._form.pack(self.desc, x, self.codes, self.scales, stream)

    def unpack(self, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        if out is None:
            if self.out is None:
                with _allocating_for(stream):
                    self.out = torch.empty(self.M, self.K, dtype=self.dtype, device=self.codes.device)
            out = self.out
        self.desc.ldx = out.stride(0) if self.M > 1 else self.K
        self._form.unpack(self.desc, self.codes, self.scales, out, stream)
        return out

    def saved_bytes(self) -> int:
        """Codes and scales."""
        return self.codes.nbytes + self.scales.nbytes


class F8Checkpoint(Checkpoint):
    """The same in 8-bit floating point: e4m3 codes with a power of two for each block of 128 channels, so that a loud channel costs none but its
    block's neighbours their bits."""

    _form = _F8Rows


def linear_workspace_bytes(M: int, K: int, N: int, dtype=torch.bfloat16, train: bool = True, gap: int = 0, form=_IntRows) -> int:
    """What `Linear` of these sizes needs as its `ws`."""
    d = B.make_qdesc(M, K, N, _dtype(dtype), K + gap, N + gap)
    return max(form.workspace_bytes(d, p) for p in ((B.PASS_FWD, B.PASS_BWD) if train else (B.PASS_FWD,)))


def f8_linear_workspace_bytes(M: int, K: int, N: int, dtype=torch.bfloat16, train: bool = True, gap: int = 0) -> int:
    """What `F8Linear` of these sizes needs as its `ws`."""
    return linear_workspace_bytes(M, K, N, dtype, train, gap, _F8Rows)


class Linear:
    """z = x w^T + b on M rows: x and w in 8 bits with a scale for each row of x and each output channel, integer sums.

    train: the codes of x are kept for `backward`, which works from them (x itself may be dropped after `forward`).
    gap: x, dx, z and dz are rows of buffers with `gap` elements between the rows.
    packed: x always comes packed (`forward_packed`), so the layer has no codes of its own.
    need_dx, need_dW: gradients that are ever asked for; there are buffers for these alone.
    z, dx: rows that the layer writes, ws: bytes that it works in (`linear_workspace_bytes`), where several layers share them."""

    _form = _IntRows

    def __init__(self, M: int, K: int, N: int, dtype=torch.bfloat16, train: bool = True, gap: int = 0, device="cuda",
                 packed: bool = False, need_dx: bool = True, need_dW: bool = True, z: Optional[torch.Tensor] = None,
                 dx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None):
        self.M, self.K, self.N, self.dtype, self.train = M, K, N, dtype, train
        self.ldx, self.ldz = K + gap, N + gap
        self.desc = B.make_qdesc(M, K, N, _dtype(dtype), self.ldx, self.ldz)
        self._add_desc = B.make_qdesc(M, K, N, _dtype(dtype), self.ldx, self.ldz)   # (with an addend)
        self.packed = packed
        self.codes, self.scales = self._form.new(M, K, device) if train and not packed else (None, None)   # what forward packs into
        self._kept = None, None   # what backward reads: these, or those that forward_packed was given
        self.w_codes = self.w_scales = None   # the weight in use
        self._own_weight = None               # what pack_weight packs into
        self._w_desc = B.make_qdesc(N, K, dtype=_dtype(dtype))
        self.z = _rows(z, M, N, self.ldz, dtype, device, "z")
        self.dx = _rows(dx, M, K, self.ldx, dtype, device, "dx") if train and need_dx else None
        self.dW = torch.empty(N, K, dtype=dtype, device=device) if train and need_dW else None
        self.db = torch.empty(N, dtype=torch.float32, device=device) if train else None
        need = linear_workspace_bytes(M, K, N, dtype, train, gap, self._form)
        if ws is not None and ws.nbytes < need:
            raise ValueError(f"ws: {ws.nbytes} bytes, {need} needed")
        self.ws = ws if ws is not None else torch.empty(need, dtype=torch.uint8, device=device) if need else None

    def set_weight(self, codes: torch.Tensor, scales: torch.Tensor):
        """A weight that is packed already (`new_codes(N, K)`, `convbn_qpack`): read where it is, never written."""
        self.w_codes, self.w_scales = _codes(codes, self.N, self.K, "codes"), self._form.scales(scales, self.N, self.K, "scales")

    def pack_weight(self, W: torch.Tensor, stream=None):
        """Pack W [N, K] by output channel, into buffers of the layer's own."""
        if self._own_weight is None:
            with _allocating_for(stream):
                self._own_weight = self._form.new(self.N, self.K, W.device)
        self._form.pack(self._w_desc, W, *self._own_weight, stream)
        self.w_codes, self.w_scales = self._own_weight

    def _desc_with(self, bit: int, field: str, add, width: int, ld: int):
        if add is None:
            return self.desc
        if (add.dtype is not self.dtype or add.shape != (self.M, width) or self.M > 1 and add.stride(0) != ld
                or self.M and width > 1 and add.stride(1) != 1 or add.device != self.z.device):
            raise ValueError(f"add: expected {self.dtype} [{self.M}, {width}] with rows {ld} elements apart on {self.z.device}")
        d = self._add_desc
        d.act = bit
        setattr(d, field, add.data_ptr())
        return d

    def _ready(self):
        if self.w_codes is None:
            raise RuntimeError("no weight: call pack_weight or set_weight first")

    def forward(self, x: torch.Tensor, b: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None, stream=None):
        """z = x w^T + b (+ add)."""
        self._ready()
        if self.packed:
            raise RuntimeError("this layer takes packed rows (packed=True)")
        if x is None:
            raise ValueError("x: expected rows")
        d = self._desc_with(B.ACT_ADD_OUT, "add_out", add, self.N, self.ldz)
        self._form.fwd(d, x, self.codes, self.scales, self.w_codes, self.w_scales, b, self.z, self.ws, stream)
        self._kept = self.codes, self.scales
        return self.z

    def forward_packed(self, codes: torch.Tensor, scales: torch.Tensor, b: Optional[torch.Tensor] = None,
                       add: Optional[torch.Tensor] = None, stream=None):
        """The same for rows that are packed already; with `train` they are what `backward` reads, so leave them as they are until then."""
        self._ready()
        if codes is None or scales is None:
            raise ValueError("codes, scales: expected packed rows")
        d = self._desc_with(B.ACT_ADD_OUT, "add_out", add, self.N, self.ldz)
        self._form.fwd(d, None, codes, scales, self.w_codes, self.w_scales, b, self.z, self.ws, stream)
        if self.train:
            self._kept = codes, scales
        return self.z

    def backward(self, dz: torch.Tensor, need_dx: Optional[bool] = None, need_dW: Optional[bool] = None, bias: bool = False,
                 add: Optional[torch.Tensor] = None, stream=None):
        """(dx (+ add), dW, db) from the kept codes; None for what is not asked for (need_dx, need_dW: as the layer was made).  bf16 dz whose N and
        row distance are multiples of 8 is read where it is, and has to start on 16 bytes."""
        if not self.train:
            raise RuntimeError("this layer keeps no codes (train=False)")
        self._ready()
        need_dx, need_dW = self.dx is not None if need_dx is None else need_dx, self.dW is not None if need_dW is None else need_dW
        if need_dx and self.dx is None or need_dW and self.dW is None:
            raise RuntimeError("this layer was made without that gradient (need_dx, need_dW)")
        d = self._desc_with(B.ACT_ADD_IN, "add_in", add, self.K, self.ldx)
        dx, dW, db = self.dx if need_dx else None, self.dW if need_dW else None, self.db if bias else None
        self._form.bwd(d, *self._kept, self.w_codes, self.w_scales, dz, dx, dW, db, self.ws, stream)
        return dx, dW, db

    def saved_bytes(self) -> int:
        """Codes and scales: what backward needs of the forward pass."""
        return self.M * (B.convbn_qrow_bytes(self.K) + self._form.scale_bytes(self.K)) if self.train else 0


class F8Linear(Linear):
    """The same block in 8-bit floating point: x and w as e4m3 codes with a power of two for each block of 128 channels of a row
    (`new_f8_codes`, `convbn_fpack`; `f8_linear_workspace_bytes`), multiplied as they are held, sums in fp32.  `backward` meets unrounded
    gradients with the values that the codes stand for, which are bf16 numbers whatever their scale."""

    _form = _F8Rows


class Gate:
    """y = f(g) u for rows h = [g | u] of 2 K channels, f = "silu" or "gelu".

    train: the codes of g and u are kept for `backward`.  packed: y comes as codes and scales (`codes_y`, `scales_y`), the form that the
    next Linear takes, and not as a tensor.  gap: as in Linear.  y, dh: rows that the gate writes, where several layers share them (dh may be
    h itself, which backward does not read)."""

    def __init__(self, M: int, K: int, dtype=torch.bfloat16, kind: str = "silu", train: bool = True, packed: bool = False, gap: int = 0,
                 device="cuda", y: Optional[torch.Tensor] = None, dh: Optional[torch.Tensor] = None):
        self.M, self.K, self.dtype = M, K, dtype
        self.ldh, self.ldy = 2 * K + gap, K + gap
        self.desc = B.make_qdesc(M, K, dtype=_dtype(dtype), ldx=self.ldh, ldz=self.ldy, gate=_GATES[kind])
        self.codes, self.scales = new_codes(2 * M, K, device) if train else (None, None)
        self.codes_y, self.scales_y = new_codes(M, K, device) if packed else (None, None)
        self.y = None if packed else _rows(y, M, K, self.ldy, dtype, device, "y")
        self.dh = _rows(dh, M, 2 * K, self.ldh, dtype, device, "dh") if train else None

    def forward(self, h: torch.Tensor, stream=None):
        B.convbn_qgate_fwd(self.desc, h, self.codes, self.scales, self.y, self.codes_y, self.scales_y, stream)
        return self.y

    def backward(self, dy: torch.Tensor, stream=None):
        if self.codes is None:
            raise RuntimeError("this gate keeps no codes (train=False)")
        B.convbn_qgate_bwd(self.desc, self.codes, self.scales, dy, self.dh, stream)
        return self.dh

    def saved_bytes(self) -> int:
        """Codes and scales of g and u."""
        return 0 if self.codes is None else self.codes.numel() + 8 * self.M


class GatedBlock:
    """out = x + down(f(up_g(x)) up_u(x)): the gated two-layer block on M rows of C channels with F hidden ones, on a backbone's last
    feature map (rows = pixels) or a token stream.  Backward needs the codes of x, h and y only; h itself is scratch, and its gradient takes
    its place.

    share: a block of the same sizes whose full-width tensors and workspace this one uses too, as the blocks of a stack do: forward then updates
    the rows that `out` goes through in place (x may be the other block's out), backward those of the gradient (dout may be the other's dx)."""

    def __init__(self, M: int, C: int, F: int, dtype=torch.bfloat16, kind: str = "silu", train: bool = True, device="cuda",
                 share: Optional["GatedBlock"] = None):
        if share is None:
            need = max(linear_workspace_bytes(M, C, 2 * F, dtype, train), linear_workspace_bytes(M, F, C, dtype, train))
            h, out, dy, dx, ws = None, None, None, None, torch.empty(need, dtype=torch.uint8, device=device) if need else None
        else:
            if train and not share.up.train:
                raise ValueError("share: a block that is not trained has no gradients to share")
            h, out, dy, dx, ws = share.up.z, share.down.z, share.down.dx, share.up.dx, share.up.ws
        self.up = Linear(M, C, 2 * F, dtype, train, device=device, z=h, dx=dx, ws=ws)
        self.gate = Gate(M, F, dtype, kind, train, packed=True, device=device, dh=self.up.z)
        self.down = Linear(M, F, C, dtype, train, device=device, packed=True, z=out, dx=dy, ws=ws)

    def pack_weights(self, W_up: torch.Tensor, W_down: torch.Tensor, stream=None):
        """W_up [2 F, C] (g's rows before u's), W_down [C, F]: once for serving, every step in training."""
        self.up.pack_weight(W_up, stream)
        self.down.pack_weight(W_down, stream)

    def forward(self, x: torch.Tensor, stream=None):
        self.gate.forward(self.up.forward(x, stream=stream), stream)
        return self.down.forward_packed(self.gate.codes_y, self.gate.scales_y, add=x, stream=stream)

    def backward(self, dout: torch.Tensor, stream=None):
        """(dx, dW_up, dW_down)."""
        dy, dW_down, _ = self.down.backward(dout, stream=stream)
        dx, dW_up, _ = self.up.backward(self.gate.backward(dy, stream), add=dout, stream=stream)
        return dx, dW_up, dW_down

    def saved_bytes(self) -> int:
        """Codes and scales of x, h and y."""
        return self.up.saved_bytes() + self.gate.saved_bytes() + self.down.saved_bytes()
