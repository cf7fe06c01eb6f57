"""Layer operators in front of the gradient compression: layer norm, 8-bit checkpoints, block-scaled 8-bit products and
per-node weight gradients (binding of the section "layer operators" of include/lgc.h: argument checks and marshalling
only).

The K nodes' tokens are K runs of rows of one activation matrix; node k has rows ``node_start[k] .. node_start[k+1]-1``.
Gradients of weights come out per node, in views of the ``[K][N]`` gradients that :meth:`lgc.LGC.accumulate` reads::

    h8 = layers.packed_empty(rows, C)
    layers.layer_norm(x, gamma, beta, 1e-5, mean, rstd, packed=h8)           # h = norm(x), in 8 bits
    layers.product(h8, w8, y=z)                                              # z = h W^T
    ...
    layers.pack(dz, dz8)
    layers.product(dz8, w8, y=dh, across=True)                               # dh = dz W, the same weight bytes
    layers.weight_gradient(dz, h8, grads[:, at:at + n], node_start=starts)   # dW of every node into its row
    layers.layer_norm_backward(dh, x, gamma, mean, rstd, dx, grads[:, g0:g1], grads[:, b0:b1], node_start=starts)

Outputs are the caller's tensors; a call enqueues on ``stream`` (default: the current stream) and returns.  With a ``stream``
of the caller's, the order against other streams and the tensors' lifetime until the stream is done (``record_stream``) are
the caller's too; scratch that a call allocates belongs to that stream.  A call runs on the current device and refuses
operands and streams of another one.
"""
from __future__ import annotations

import contextlib
import ctypes as C
from typing import Optional, Union

import torch

from . import lgc
from .lgc import LGC_OK, LGCError

BLOCK = 128
TYPE_FP32, TYPE_BF16, TYPE_PACKED = 0, 1, 2
_TYPES = {torch.float32: TYPE_FP32, torch.bfloat16: TYPE_BF16}


class Packed:
    """An 8-bit matrix: e4m3 `codes` (uint8 [rows][ld], unit column stride, 16-byte aligned rows) and the blocks' scale
    bytes (uint8 [ceil(rows / block_rows)][..], read four at a time); `cols` of the codes' columns belong to it."""

    __slots__ = ("codes", "scales", "rows", "cols", "block_rows", "device_index", "_c")

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, cols: Optional[int] = None, block_rows: int = 1):
        if not (codes.is_cuda and scales.get_device() == codes.get_device() and codes.dtype is torch.uint8 and scales.dtype is torch.uint8):
            raise ValueError("codes and scales: need 2-D uint8 CUDA tensors of one device")
        shape, tall, ld, lds = codes.shape, scales.shape, codes.stride(), scales.stride()
        if len(shape) != 2 or len(tall) != 2:
            raise ValueError("codes and scales: need 2-D uint8 CUDA tensors")
        rows, width = shape
        if cols is None:
            cols = width
        if block_rows != 1 and block_rows != BLOCK:
            raise ValueError("block_rows: 1 or 128")
        if not (0 < cols <= width and ld[1] == 1 and lds[1] == 1 and tall[0] == -(-rows // block_rows) and tall[1] * BLOCK >= cols):
            raise ValueError("codes need unit column stride and `cols` columns, scales a row per row of blocks and a byte per block")
        self.codes, self.scales, self.rows, self.cols, self.block_rows = codes, scales, rows, cols, block_rows
        self.device_index = codes.get_device()
        # (the row stride of a tensor with one row may be anything)
        self._c = lgc.lgc_packed(codes.data_ptr(), ld[0] if rows > 1 else -(-width // 16) * 16,
                                 scales.data_ptr(), lds[0] if tall[0] > 1 else -(-tall[1] // 4) * 4)


def packed_empty(rows: int, cols: int, block_rows: int = 1, device: Optional[torch.device] = None) -> Packed:
    """Room for an 8-bit matrix, its rows padded to what the calls need."""
    dev = device if device is not None else torch.device("cuda")
    return Packed(torch.empty(rows, -(-cols // 16) * 16, dtype=torch.uint8, device=dev),
                  torch.empty(-(-rows // block_rows), -(-cols // (4 * BLOCK)) * 4, dtype=torch.uint8, device=dev), cols, block_rows)


def _device(index: int, stream: Optional[torch.cuda.Stream]) -> int:
    """The device that a call runs on, given its first operand's: the current one, since the library launches there."""
    if index < 0:
        raise ValueError("need CUDA tensors")
    current = torch._C._cuda_getDevice()
    if index != current:
        raise ValueError(f"the operands are on cuda:{index}, the current device is cuda:{current} (set it with torch.cuda.device)")
    if stream is not None and stream.device_index != index:
        raise ValueError(f"stream: of cuda:{stream.device_index}, the operands are on cuda:{index}")
    return index


def _stream(stream: Optional[torch.cuda.Stream], device: int) -> int:
    # (torch.cuda.current_stream builds a Stream object: 2 us, as much as the launch)
    return torch._C._cuda_getCurrentRawStream(device) if stream is None else stream.cuda_stream


def _matrix(t: torch.Tensor, name: str, device: int, want: Optional[tuple] = None):
    """(rows, columns, row stride, type) of a matrix argument, after the checks that need the tensor (the library checks the
    numbers)."""
    shape, kind = t.shape, _TYPES.get(t.dtype)
    if kind is None or len(shape) != 2 or t.get_device() != device:
        raise ValueError(f"{name}: need a 2-D fp32 or bf16 tensor with unit column stride on cuda:{device}")
    ld, unit = t.stride()
    rows, cols = shape
    if unit != 1 and cols > 1:
        raise ValueError(f"{name}: need a 2-D fp32 or bf16 tensor with unit column stride on cuda:{device}")
    if want is not None and (rows, cols) != want:
        raise ValueError(f"{name}: need {want[0]} x {want[1]} elements, got {rows} x {cols}")
    # a single row may have any stride: report one that the library accepts
    return rows, cols, (ld if rows > 1 else -(-cols // 8) * 8), kind


def _vector(t: torch.Tensor, n: int, name: str, device: int) -> int:
    if not (t.dtype is torch.float32 and t.get_device() == device and t.numel() == n and t.is_contiguous()):
        raise ValueError(f"{name}: need a contiguous fp32 tensor of {n} elements on cuda:{device}")
    return t.data_ptr()


def _packed(p: Packed, name: str, device: int, rows: int, cols: int, block_rows: int = 1):
    if p.device_index != device:
        raise ValueError(f"{name}: need an 8-bit matrix on cuda:{device}")
    if p.rows != rows or p.cols != cols or p.block_rows != block_rows:
        raise ValueError(f"{name}: need a {rows} x {cols} 8-bit matrix with block_rows {block_rows}, got {p.rows} x {p.cols}, {p.block_rows}")
    return C.byref(p._c)


def _nodes(node_start: Optional[torch.Tensor], out: torch.Tensor, n: int, name: str, device: int):
    """(pointer to node_start, number of nodes, node stride) for per-node results in `out` [K][n]."""
    if not (out.get_device() == device and out.dtype == torch.float32 and out.dim() == 2 and out.shape[1] == n and (n == 1 or out.stride(1) == 1)):
        raise ValueError(f"{name}: need a [nodes][{n}] fp32 view with unit column stride on cuda:{device}")
    K = out.shape[0]
    if node_start is None:
        if K != 1:
            raise ValueError("node_start: needed with more than one node")
        return None, 1, n
    if not (node_start.get_device() == device and node_start.dtype == torch.int64 and node_start.is_contiguous() and node_start.numel() == K + 1):
        raise ValueError(f"node_start: need a contiguous int64 tensor of {K + 1} elements on cuda:{device}")
    return node_start.data_ptr(), K, (out.stride(0) if K > 1 else n)


def _done(status: int, where: str) -> None:
    if status != LGC_OK:
        raise LGCError(status, where, lgc.lib().lgc_last_error(None).decode())


def pack(x: torch.Tensor, out: Packed, slope: float = 1.0, gate: Optional[Packed] = None, y: Optional[torch.Tensor] = None,
         stream: Optional[torch.cuda.Stream] = None) -> None:
    """`x` (fp32 or bf16), through a leaky ReLU of `slope` (1: none), to 8 bits.  With `gate` (the 8-bit result of that
    leaky ReLU, `slope` not negative) `x` is a gradient and gets its derivative instead.  `y` (bf16): also what was rounded."""
    device = _device(x.get_device(), stream)
    rows, cols, ldx, kind = _matrix(x, "x", device)
    yp = ldy = None
    if y is not None:
        _, _, ldy, ykind = _matrix(y, "y", device, (rows, cols))
        if ykind != TYPE_BF16:
            raise ValueError("y: need a bf16 tensor")
        yp = y.data_ptr()
    _done(lgc.lib().lgc_pack(x.data_ptr(), kind, rows, cols, ldx, out.block_rows, slope,
                             None if gate is None else _packed(gate, "gate", device, rows, cols),
                             _packed(out, "out", device, rows, cols, out.block_rows), yp, ldy or 0, _stream(stream, device)), "lgc_pack")


def unpack(src: Packed, y: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> None:
    """The values of an 8-bit matrix in `y` (fp32 or bf16; exact in both)."""
    device = _device(src.device_index, stream)
    rows, cols, ldy, kind = _matrix(y, "y", device, (src.rows, src.cols))
    _done(lgc.lib().lgc_unpack(C.byref(src._c), rows, cols, src.block_rows, y.data_ptr(), kind, ldy, _stream(stream, device)), "lgc_unpack")


def layer_norm(x: torch.Tensor, gamma: torch.Tensor, beta: torch.Tensor, eps: float, mean: torch.Tensor, rstd: torch.Tensor,
               y: Optional[torch.Tensor] = None, packed: Optional[Packed] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Layer norm of the rows of `x` into `y` (x's type) and / or, in 8 bits, `packed`; `mean` and `rstd` for the backward pass."""
    device = _device(x.get_device(), stream)
    rows, cols, ldx, kind = _matrix(x, "x", device)
    yp = ldy = None
    if y is not None:
        _, _, ldy, ykind = _matrix(y, "y", device, (rows, cols))
        if ykind != kind:
            raise ValueError("y: need x's type")
        yp = y.data_ptr()
    _done(lgc.lib().lgc_layer_norm(x.data_ptr(), kind, rows, cols, ldx, _vector(gamma, cols, "gamma", device), _vector(beta, cols, "beta", device),
                                   eps, yp, ldy or 0, None if packed is None else _packed(packed, "packed", device, rows, cols),
                                   _vector(mean, rows, "mean", device), _vector(rstd, rows, "rstd", device), _stream(stream, device)), "lgc_layer_norm")


def layer_norm_backward_scratch(rows: int, cols: int, num_nodes: int = 1) -> int:
    """Bytes of scratch that layer_norm_backward needs."""
    n = C.c_size_t()
    _done(lgc.lib().lgc_layer_norm_backward_scratch(rows, cols, num_nodes, C.byref(n)), "lgc_layer_norm_backward_scratch")
    return n.value


def _scratch(need: int, scratch: Optional[torch.Tensor], stream: Optional[torch.cuda.Stream], like: torch.Tensor):
    """(tensor, bytes) of a call's scratch: the caller's, or from PyTorch's allocator."""
    if scratch is None:
        # of the pool of the stream that uses it: in another pool's block earlier work of that pool's stream may be under way
        with torch.cuda.stream(stream) if stream is not None else contextlib.nullcontext():
            return torch.empty(need, dtype=torch.uint8, device=like.device), need
    if not (scratch.get_device() == like.get_device() and scratch.dtype is torch.uint8 and scratch.is_contiguous()):
        raise ValueError(f"scratch: need a contiguous uint8 tensor on cuda:{like.get_device()}")
    return scratch, scratch.numel()


def layer_norm_backward(dy: torch.Tensor, x: Union[torch.Tensor, Packed], gamma: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        dx: torch.Tensor, dgamma: torch.Tensor, dbeta: torch.Tensor, node_start: Optional[torch.Tensor] = None,
                        scratch: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """Backward pass of layer_norm.  `x`: the input, or its 8-bit checkpoint.  `dgamma`, `dbeta`: [nodes][cols] views with
    one row stride (columns of the nodes' gradients); rows in no node's run get their `dx` too.  `scratch`: a uint8 tensor of
    layer_norm_backward_scratch bytes; without one it comes from PyTorch's allocator."""
    device = _device(dy.get_device(), stream)
    rows, cols, ld_dy, kind = _matrix(dy, "dy", device)
    _, _, ld_dx, dx_kind = _matrix(dx, "dx", device, (rows, cols))
    if dx_kind != kind:
        raise ValueError("dx: need dy's type")
    nodes = _nodes(node_start, dgamma, cols, "dgamma", device)
    if _nodes(node_start, dbeta, cols, "dbeta", device) != nodes:
        raise ValueError("dgamma and dbeta: need the same nodes and row stride")
    start, K, stride = nodes
    if isinstance(x, Packed):
        xp, ldx, xkind, x8 = None, 0, TYPE_PACKED, _packed(x, "x", device, rows, cols)
    else:
        _, _, ldx, xkind = _matrix(x, "x", device, (rows, cols))
        xp, x8 = x.data_ptr(), None
    scratch, size = _scratch(layer_norm_backward_scratch(rows, cols, K), scratch, stream, dy)
    _done(lgc.lib().lgc_layer_norm_backward(
        dy.data_ptr(), kind, ld_dy, xp, xkind, ldx, x8, rows, cols, _vector(gamma, cols, "gamma", device), _vector(mean, rows, "mean", device),
        _vector(rstd, rows, "rstd", device), start, K, dx.data_ptr(), ld_dx, dgamma.data_ptr(), dbeta.data_ptr(), stride, scratch.data_ptr(), size,
        _stream(stream, device)), "lgc_layer_norm_backward")


def product(a: Packed, b: Packed, y: Optional[torch.Tensor] = None, packed: Optional[Packed] = None, across: bool = False,
            slope: float = 1.0, stream: Optional[torch.cuda.Stream] = None) -> None:
    """act(a b^T), or with `across` act(a b), of 8-bit matrices (`b`: weights, block_rows 128) into `y` (fp32 or bf16) and / or,
    in 8 bits, `packed`.  act: the leaky ReLU of `slope` (1: none)."""
    device = _device(a.device_index, stream)
    rows, inner = a.rows, a.cols
    cols = b.cols if across else b.rows
    ap = _packed(a, "a", device, rows, inner)
    bp = _packed(b, "b", device, inner if across else cols, cols if across else inner, BLOCK)
    yp, ldy, kind = None, 0, TYPE_BF16
    if y is not None:
        _, _, ldy, kind = _matrix(y, "y", device, (rows, cols))
        yp = y.data_ptr()
    _done(lgc.lib().lgc_product(ap, bp, 1 if across else 0, rows, cols, inner, slope, yp, kind, ldy,
                                None if packed is None else _packed(packed, "packed", device, rows, cols), _stream(stream, device)), "lgc_product")


def weight_gradient_scratch(rows: int, cols: int, inner: int, num_nodes: int = 1) -> int:
    """Bytes of scratch that weight_gradient needs."""
    n = C.c_size_t()
    _done(lgc.lib().lgc_weight_gradient_scratch(rows, cols, inner, num_nodes, C.byref(n)), "lgc_weight_gradient_scratch")
    return n.value


def weight_gradient(dy: torch.Tensor, x: Packed, dw: torch.Tensor, node_start: Optional[torch.Tensor] = None,
                    scratch: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """dw[k] = the sum over node k's rows of dy^T x ([dy's columns][x's columns], flat), from the bf16 gradient `dy` (rows
    16-byte aligned) and the 8-bit checkpoint `x`.  `dw`: a [nodes][n] fp32 view (columns of the nodes' gradients).
    `scratch`: a uint8 tensor of weight_gradient_scratch bytes; without one it comes from PyTorch's allocator."""
    device = _device(dy.get_device(), stream)
    rows, cols, ld_dy, kind = _matrix(dy, "dy", device)
    if kind != TYPE_BF16:
        raise ValueError("dy: need a bf16 tensor")
    inner = x.cols
    xp = _packed(x, "x", device, rows, inner)
    start, K, stride = _nodes(node_start, dw, cols * inner, "dw", device)
    scratch, size = _scratch(weight_gradient_scratch(rows, cols, inner, K), scratch, stream, dy)
    _done(lgc.lib().lgc_weight_gradient(dy.data_ptr(), ld_dy, xp, rows, cols, inner, start, K, dw.data_ptr(), stride, scratch.data_ptr(), size,
                                        _stream(stream, device)), "lgc_weight_gradient")


def check(stream: Optional[torch.cuda.Stream] = None) -> None:
    """Waits for the stream and raises if a kernel recorded a failure (a wait that ran out).  One record per device and
    process: whoever checks first hears of it, and clears it."""
    s = stream if stream is not None else torch.cuda.current_stream()
    _device(s.device_index, None)
    _done(lgc.lib().lgc_layers_check(s.cuda_stream), "lgc_layers_check")
