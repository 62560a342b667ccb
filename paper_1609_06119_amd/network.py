"""Operators of a network on binned events, beside the forest (include/fbdt.h,
"A network on binned events"): tokens of the bin codes, the lookup of their
vectors and its gradient, the norm with the residual's addition and its
gradient, rows packed in 8 bits, and the products of packed rows with the
gradient of their weights.

Argument marshalling only, as in api.py: every operator is a kernel of libfbdt
on the current HIP stream, and all its tensors are on the current device.  Float
matrices are float32, bfloat16 or float16 with unit stride along columns; leading
dimensions count as rows where they can be viewed as one.

`out`, where a call takes it, must not overlap what the call reads.

The calls build no graph of torch's: gradients are calls of their own, and a tensor
that requires grad is refused while torch records gradients.
"""
from __future__ import annotations

import dataclasses
import math
import typing

import torch

from ._lib import check, lib
from .api import Codes

__all__ = ["Packed", "Normed", "event_tokens", "embed", "embed_grad", "rms_norm", "rms_norm_grad",
           "pack", "packed_product", "packed_weight_grad"]

BLOCK = 128   # columns that share a scale
_E4M3, _E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


_current_device = getattr(torch._C, "_cuda_getDevice", None)           # (None without HIP)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor) -> int:
    """The current HIP stream of the tensor's device."""
    return _raw_stream(t.get_device())


def _type(t: torch.Tensor, name: str) -> int:
    code = _TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, bfloat16 or float16, got {t.dtype}")
    return code


def _on_gpu(t, name: str):
    at = t.get_device() if isinstance(t, torch.Tensor) else -1      # (-1: on the host)
    if at >= 0 and at == _current_device():
        if t.requires_grad and torch.is_grad_enabled():
            raise ValueError(f"{name} requires grad, which the call would not record: call it under "
                             f"torch.no_grad() and take gradients from the *_grad calls")
        return
    if at < 0:
        raise TypeError(f"{name} must be a CUDA (HIP) tensor")
    raise ValueError(f"{name} is on {t.device}, the current device is cuda:{_current_device()}")


def _rows(t: torch.Tensor, name: str, dtype=None):
    """(pointer, rows, width, row stride) of t as a matrix with unit stride along columns."""
    _on_gpu(t, name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.dim() != 2:
        if t.dim() == 0:
            raise ValueError(f"{name} must have a dimension of columns")
        try:
            t = t.view(math.prod(t.shape[:-1]), t.shape[-1])
        except RuntimeError:
            raise ValueError(f"{name}: its leading dimensions cannot be viewed as rows") from None
    rows, width = t.shape
    ld, step = t.stride()
    if step != 1 and width > 1 and rows > 0:
        raise ValueError(f"{name} must have unit stride along columns")
    if rows <= 1:
        ld = width               # (a single row may report any stride)
    elif ld < width:
        raise ValueError(f"{name}: rows overlap (stride {ld}, width {width})")
    return t.data_ptr(), rows, width, ld


def _vector(t, name: str, numel: int):
    _on_gpu(t, name)
    if t.dtype != torch.float32:
        raise TypeError(f"{name} must be torch.float32, got {t.dtype}")
    if t.dim() != 1 or t.numel() != numel or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous with {numel} elements")


def _same(t: torch.Tensor, like: torch.Tensor, name: str):
    if t.shape != like.shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, needs {tuple(like.shape)}")


def _work(bytes_: int, like: torch.Tensor):
    """Workspace of a call: from torch's allocator, on the current stream."""
    return like.new_empty(bytes_, dtype=torch.uint8) if bytes_ > 0 else None


def _like(t: torch.Tensor) -> torch.Tensor:
    """An empty tensor of t's shape, type and device, without gaps between its rows."""
    if t.is_contiguous():
        return torch.empty_like(t)          # (half the time of the other)
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _ptr(t):
    return t.data_ptr() if t is not None else None


@dataclasses.dataclass
class Packed:
    """Rows in 8 bits: codes float8_e4m3fn [rows][ld] (ld a multiple of 128 and
    >= width) and a power-of-two scale per row and block of 128 columns,
    float8_e8m0fnu [rows][lds] (lds a multiple of 4).  What the columns and
    blocks beyond the width hold never influences a result."""

    data: torch.Tensor
    scales: torch.Tensor
    width: int

    @property
    def rows(self) -> int:
        return int(self.data.shape[0])

    @staticmethod
    def empty(rows: int, width: int, device="cuda") -> "Packed":
        blocks = -(-width // BLOCK)
        return Packed(torch.empty((rows, blocks * BLOCK), dtype=_E4M3, device=device),
                      torch.empty((rows, (blocks + 3) & ~3), dtype=_E8M0, device=device), width)

    def unpack(self, dtype=torch.float32) -> torch.Tensor:
        """The values [rows][width] (for inspection: elementary torch operations)."""
        blocks = -(-self.width // BLOCK)
        v = self.data[:, : blocks * BLOCK].float().reshape(self.rows, blocks, BLOCK)
        v = v * self.scales[:, :blocks].float()[:, :, None]
        return v.reshape(self.rows, -1)[:, : self.width].to(dtype)


def _packed(p: Packed, name: str):
    """(codes pointer, stride, scales pointer, stride, rows, width) of packed rows."""
    if not isinstance(p, Packed):
        raise TypeError(f"{name} must be Packed")
    d, s, width = p.data, p.scales, p.width
    _on_gpu(d, name)
    _on_gpu(s, name)
    if d.dtype != _E4M3 or s.dtype != _E8M0:
        raise TypeError(f"{name} must hold float8_e4m3fn codes and float8_e8m0fnu scales")
    try:
        (ld, step), (lds, sstep), (rows, held), (srows, sheld) = d.stride(), s.stride(), d.shape, s.shape
    except ValueError:
        raise ValueError(f"{name}: codes and scales must be matrices") from None
    blocks = (width + BLOCK - 1) // BLOCK
    if rows != srows or width < 1 or held < blocks * BLOCK or sheld < blocks:
        raise ValueError(f"{name}: codes {tuple(d.shape)} and scales {tuple(s.shape)} do not hold "
                         f"rows of width {width}")
    if rows > 0 and (step != 1 or (sstep != 1 and sheld > 1)):
        raise ValueError(f"{name}: codes and scales must have unit stride along columns")
    if rows <= 1:               # (a single row may report any stride)
        ld, lds = (held + BLOCK - 1) // BLOCK * BLOCK, (sheld + 3) & ~3
    return d.data_ptr(), ld, s.data_ptr(), lds, rows, width


class Normed(typing.NamedTuple):
    """What rms_norm returns: y (a tensor, or Packed), h = x + residual (x itself
    without a residual), and rstd float32, one per row."""

    y: typing.Any
    h: torch.Tensor
    rstd: torch.Tensor


def event_tokens(codes: Codes, n_bins: int, out: torch.Tensor | None = None) -> torch.Tensor:
    """Tokens int32 [n][d] of binned events: feature * n_bins + code, -1 (masked)
    for a missing value."""
    data, n = codes.data, codes.n
    _on_gpu(data, "codes")
    if data.dtype != torch.uint8 or data.dim() != 2 or data.stride(1) != 1:
        raise ValueError("codes must be uint8 [d][ldb] with unit stride along events")
    d, ldb = data.shape[0], data.stride(0)
    if n > ldb:
        raise ValueError(f"codes hold {ldb} events, not {n}")
    if out is None:
        out = torch.empty((n, d), dtype=torch.int32, device=data.device)
    else:
        _on_gpu(out, "out")
        if out.dtype != torch.int32 or out.shape != (n, d) or not out.is_contiguous():
            raise ValueError(f"out must be contiguous int32 [{n}][{d}]")
    check("fbdt_event_tokens", lib().fbdt_event_tokens(data.data_ptr(), n, d, ldb, n_bins,
                                                       out.data_ptr(), _stream(out)))
    return out


def _tokens(tokens: torch.Tensor) -> int:
    _on_gpu(tokens, "tokens")
    if tokens.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"tokens must be int32 or int64, got {tokens.dtype}")
    if not tokens.is_contiguous():
        raise ValueError("tokens must be contiguous")
    return 4 if tokens.dtype == torch.int32 else 8


def embed(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0,
          out: torch.Tensor | None = None) -> torch.Tensor:
    """scale * table[tokens], shape [*tokens.shape][width], of the table's type;
    tokens outside the table are masked and give zeros."""
    pt, rows, width, ldt = _rows(table, "table")
    code, size = _type(table, "table"), _tokens(tokens)
    shape = (*tokens.shape, width)
    if out is None:
        out = table.new_empty(shape)
        po, ldo = out.data_ptr(), width
    else:
        if out.shape != shape:
            raise ValueError(f"out has shape {tuple(out.shape)}, needs {shape}")
        po, _, _, ldo = _rows(out, "out", table.dtype)
    check("fbdt_embed", lib().fbdt_embed(pt, code, rows, width, ldt, tokens.data_ptr(), size,
                                         tokens.numel(), scale, po, ldo, _stream(out)))
    return out


def embed_grad(tokens: torch.Tensor, dout: torch.Tensor, rows: int, scale: float = 1.0,
               dtype: torch.dtype = torch.float32, out: torch.Tensor | None = None) -> torch.Tensor:
    """Gradient [rows][width] of embed's table for dout [*tokens.shape][width]:
    float32, or of dout's type.  Sums are float32 in the order of the positions."""
    size, n = _tokens(tokens), tokens.numel()
    if dout.shape[:-1] != tokens.shape:
        raise ValueError(f"dout has shape {tuple(dout.shape)}, tokens {tuple(tokens.shape)}")
    code, width = _type(dout, "dout"), dout.shape[-1]
    _on_gpu(dout, "dout")
    pd, ldd = dout.data_ptr(), width
    if n:
        pd, _, _, ldd = _rows(dout, "dout")
    out = _result(out, (int(rows), width), dtype, dout)
    po, _, _, ldo = _rows(out, "out", dtype)
    L = lib()
    need = L.fbdt_embed_grad_work(n, int(rows), width)
    work = _work(need, dout)
    check("fbdt_embed_grad",
          L.fbdt_embed_grad(tokens.data_ptr(), size, n, pd, code, ldd, scale, po, _type(out, "out"),
                            int(rows), width, ldo, _ptr(work), need, _stream(out)))
    return out


def rms_norm(x: torch.Tensor, gain: torch.Tensor, eps: float = 1e-6,
             residual: torch.Tensor | None = None, packed: bool = False) -> Normed:
    """Root-mean-square norm of the rows of h = x + residual: y = h * rstd * gain
    with rstd = 1 / sqrt(mean(h^2) + eps); packed: y in 8 bits with scales."""
    px, n, width, ldx = _rows(x, "x")
    code = _type(x, "x")
    _vector(gain, "gain", width)
    pr, ldr, ph, h = None, 0, None, x
    if residual is not None:
        _same(residual, x, "residual")
        pr, _, _, ldr = _rows(residual, "residual", x.dtype)
        h = _like(x)
        ph = h.data_ptr()
    rstd = gain.new_empty(n)
    if packed:
        y = Packed.empty(n, width, x.device)
        out = (None, width, y.data.data_ptr(), y.data.shape[1], y.scales.data_ptr(),
               y.scales.shape[1])
    else:
        y = _like(x)
        out = (y.data_ptr(), width, None, 0, None, 0)
    check("fbdt_rms_norm",
          lib().fbdt_rms_norm(px, ldx, pr, ldr, code, n, width, gain.data_ptr(), eps, ph, width, *out,
                              rstd.data_ptr(), _stream(x)))
    return Normed(y, h, rstd)


def rms_norm_grad(dy: torch.Tensor, h: torch.Tensor, gain: torch.Tensor, rstd: torch.Tensor,
                  dh: torch.Tensor | None = None):
    """(dx, dgain) of rms_norm from the gradient of y, the h and rstd of the
    forward call and, if there is one, the gradient dh of h.  dx (of h's type)
    is the gradient of x and of the residual; dgain is float32."""
    ph, n, width, ldh = _rows(h, "h")
    code = _type(h, "h")
    _same(dy, h, "dy")
    pd, _, _, ldd = _rows(dy, "dy", h.dtype)
    _vector(gain, "gain", width)
    _vector(rstd, "rstd", n)
    pu, ldu = None, 0
    if dh is not None:
        _same(dh, h, "dh")
        pu, _, _, ldu = _rows(dh, "dh", h.dtype)
    dx = _like(h)
    dgain = torch.empty_like(gain)
    L = lib()
    need = L.fbdt_rms_norm_grad_work(n, width)
    work = _work(need, h)
    check("fbdt_rms_norm_grad",
          L.fbdt_rms_norm_grad(pd, ldd, ph, ldh, pu, ldu, code, n, width, gain.data_ptr(),
                               rstd.data_ptr(), dx.data_ptr(), width, dgain.data_ptr(), _ptr(work),
                               need, _stream(h)))
    return dx, dgain


def pack(x: torch.Tensor) -> Packed:
    """The rows of x in 8 bits with a power-of-two scale for each block of 128 columns."""
    px, n, width, ldx = _rows(x, "x")
    code = _type(x, "x")
    p = Packed.empty(n, width, x.device)
    check("fbdt_pack", lib().fbdt_pack(px, ldx, code, n, width, p.data.data_ptr(), p.data.shape[1],
                                       p.scales.data_ptr(), p.scales.shape[1], _stream(x)))
    return p


def _result(out, shape, dtype, like: torch.Tensor):
    """out, or an empty tensor on the device of `like`."""
    if out is None:
        return like.new_empty(shape, dtype=dtype)
    if out.shape != shape:
        raise ValueError(f"out has shape {tuple(out.shape)}, needs {shape}")
    return out


def packed_product(a: Packed, b: Packed, dtype: torch.dtype = torch.bfloat16,
                   out: torch.Tensor | None = None, fast: bool = False) -> torch.Tensor:
    """a b^T, [a.rows][b.rows]: activations (or a gradient) times weights, both packed
    along the width that is summed; added in float32 and rounded once.  fast: more than
    a few rows are added by the 8-bit matrix unit, about twice as fast, to about 1.5e-5 of
    the result's norm on normal data (products are cut off 2^-13 below the largest of
    their group of 8): enough for a 16-bit result, though a single one that cancels may be
    off by more than its own rounding."""
    pa, lda, sa, ldsa, m, k = _packed(a, "a")
    pb, ldb, sb, ldsb, n, kb = _packed(b, "b")
    if k != kb:
        raise ValueError(f"widths differ: {k} and {kb}")
    out = _result(out, (m, n), dtype, a.data)
    po, _, _, ldo = _rows(out, "out", dtype)
    check("fbdt_packed_product",
          lib().fbdt_packed_product(pa, lda, sa, ldsa, m, pb, ldb, sb, ldsb, n, k, po,
                                    _type(out, "out"), ldo, fast, _stream(out)))
    return out


def packed_weight_grad(dy: torch.Tensor, x: Packed, dtype: torch.dtype = torch.float32,
                       out: torch.Tensor | None = None) -> torch.Tensor:
    """dy^T x, [dy columns][x.width]: the gradient of packed_product's weights from the
    gradient of its result (bfloat16) and the packed activations of the forward pass."""
    pd, m, n, ldd = _rows(dy, "dy", torch.bfloat16)
    px, ldx, sx, ldsx, rows, k = _packed(x, "x")
    if rows != m:
        raise ValueError(f"dy has {m} rows, x {rows}")
    out = _result(out, (n, k), dtype, dy)
    po, _, _, ldo = _rows(out, "out", dtype)
    L = lib()
    need = L.fbdt_packed_weight_grad_work(pd, ldd, m, n, k)
    work = _work(need, dy)
    check("fbdt_packed_weight_grad",
          L.fbdt_packed_weight_grad(pd, ldd, m, n, px, ldx, sx, ldsx, k, po, _type(out, "out"), ldo,
                                    _ptr(work), need, _stream(out)))
    return out
