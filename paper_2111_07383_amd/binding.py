"""Thin PyTorch binding of the C ABI: device memory and streams come from torch,
every step of the computation runs in the HIP library.

Names follow the C entry points (``ssconv_build_rulebook`` -> ``build_rulebook``
etc.).  Tensors must live on the current HIP device; bf16 tensors map to
SSCONV_BF16 and fp32 tensors to SSCONV_F32.
"""
import ctypes
from contextlib import nullcontext
from ctypes import byref, c_float, c_int, c_int64, c_void_p
from dataclasses import dataclass
from functools import lru_cache
from typing import Optional, Sequence, Tuple, Union

import numpy as np
import torch

from ._abi import BF16, F32, MAX_ENTRIES, BasisDesc, Fields, Rows, check, lib

FieldList = Sequence[Tuple[int, int]]


def _stream(stream=None) -> c_void_p:
    s = torch.cuda.current_stream() if stream is None else stream
    return c_void_p(s.cuda_stream)


def _ptr(t: Optional[torch.Tensor]) -> c_void_p:
    return c_void_p(0 if t is None else t.data_ptr())


def _dtype(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _need(t: torch.Tensor, name: str, dtype=None, shape=None):
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def make_fields(fields: FieldList) -> Fields:
    f = Fields()
    f.n = len(fields)
    for e, (l, m) in enumerate(fields):
        f.l[e] = int(l)
        f.mult[e] = int(m)
    return f


def n_channels(fields: FieldList) -> int:
    return sum(m * (2 * l + 1) for l, m in fields)


def basis_desc(fields_in: FieldList, fields_out: FieldList, ksize: int, shells: Sequence[float],
               eps: float = 0.6, jmax: Optional[int] = None) -> BasisDesc:
    d = BasisDesc()
    d.in_ = make_fields(fields_in)
    d.out = make_fields(fields_out)
    d.ksize = int(ksize)
    d.n_shells = len(shells)
    for i, m in enumerate(shells):
        d.shells[i] = float(m)
    d.eps = float(eps)
    d.jmax = -1 if jmax is None else int(jmax)
    return d


def layer_desc(layer) -> BasisDesc:
    """Descriptor of a layer spec with fields_in/out, ksize, shells, eps, jmax attributes."""
    return basis_desc(layer.fields_in, layer.fields_out, layer.ksize, layer.shells, layer.eps, layer.jmax)


def basis_info(desc: BasisDesc) -> Tuple[int, int]:
    floats, ncoef = c_int64(), c_int64()
    check(lib().ssconv_basis_info(byref(desc), byref(floats), byref(ncoef)), "ssconv_basis_info")
    return floats.value, ncoef.value


def basis_build(desc: BasisDesc) -> np.ndarray:
    """Host-built basis (fp32 numpy, layout of ssconv_basis_build)."""
    n, _ = basis_info(desc)
    out = np.zeros(max(n, 1), np.float32)
    check(lib().ssconv_basis_build(byref(desc), out.ctypes.data_as(c_void_p)), "ssconv_basis_build")
    return out[:n]


class Rulebook:
    """Owner of an ssconv_rulebook_t (hash tables, neighbour map, pair lists).

    ``asynchronous``: ssconv_build_rulebook_async -- a submanifold build returns before its pair
    counts reach the host; ``pair_counts`` / ``n_pairs`` (and ``wait()``) settle it, and so does
    every library call that needs them."""

    def __init__(self, coords: torch.Tensor, grid, ksize: int, stride: int = 1, submanifold: bool = True,
                 stream=None, asynchronous: bool = False):
        _need(coords, "coords", torch.int32)
        if coords.dim() != 2 or coords.shape[1] != 4:
            raise ValueError("coords must be [n, 4] (b, x, y, z)")
        g = (c_int * 3)(*([int(grid)] * 3 if np.isscalar(grid) else [int(v) for v in grid]))
        h = c_void_p()
        self._h = None
        self.device = coords.device
        build = lib().ssconv_build_rulebook_async if asynchronous else lib().ssconv_build_rulebook
        check(build(_ptr(coords), coords.shape[0], g, int(ksize), int(stride), int(bool(submanifold)),
                    _stream(stream), byref(h)), "ssconv_build_rulebook")
        self._h = h
        self.ksize, self.K, self.stride, self.submanifold = ksize, ksize ** 3, stride, bool(submanifold)
        self._counts = None
        self.n_in = int(coords.shape[0])
        if self.submanifold:
            self.n_out = self.n_in
        else:
            self._settle()
        if not asynchronous:
            self._settle()

    def _settle(self):
        if self._counts is None:
            n_in, n_out = c_int64(), c_int64()
            counts = (c_int64 * self.K)()
            check(lib().ssconv_rulebook_info(self.handle, byref(n_in), byref(n_out), counts), "ssconv_rulebook_info")
            self.n_in, self.n_out = n_in.value, n_out.value
            self._counts = np.array(counts[:], np.int64)
        return self._counts

    def wait(self):
        """Settles an asynchronous build (raises its error, if any)."""
        check(lib().ssconv_rulebook_wait(self.handle), "ssconv_rulebook_wait")

    @property
    def pair_counts(self) -> np.ndarray:
        return self._settle()

    @property
    def n_pairs(self) -> int:
        return int(self._settle().sum())

    @property
    def handle(self) -> c_void_p:
        if self._h is None:
            raise RuntimeError("rule book has been destroyed")
        return self._h

    def out_coords(self, stream=None) -> torch.Tensor:
        t = torch.empty((self.n_out, 4), dtype=torch.int32, device=self.device)
        check(lib().ssconv_rulebook_out_coords(self.handle, _ptr(t), _stream(stream)), "ssconv_rulebook_out_coords")
        return t

    def pairs(self, stream=None) -> torch.Tensor:
        t = torch.empty((self.n_pairs, 2), dtype=torch.int32, device=self.device)
        check(lib().ssconv_rulebook_pairs(self.handle, _ptr(t), _stream(stream)), "ssconv_rulebook_pairs")
        return t

    def neighbours(self, stream=None) -> torch.Tensor:
        t = torch.empty((self.K, self.n_out), dtype=torch.int32, device=self.device)
        check(lib().ssconv_rulebook_neighbours(self.handle, _ptr(t), _stream(stream)), "ssconv_rulebook_neighbours")
        return t

    def hash_slots(self, which: int = 0, stream=None) -> torch.Tensor:
        cap = c_int64()
        check(lib().ssconv_rulebook_hash(self.handle, which, None, byref(cap), _stream(stream)), "ssconv_rulebook_hash")
        t = torch.empty((cap.value,), dtype=torch.int64, device=self.device)
        check(lib().ssconv_rulebook_hash(self.handle, which, _ptr(t), byref(cap), _stream(stream)),
              "ssconv_rulebook_hash")
        return t

    def close(self):
        if self._h is not None:
            lib().ssconv_rulebook_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def build_rulebook(coords, grid, ksize, stride=1, submanifold=True, stream=None) -> Rulebook:
    return Rulebook(coords, grid, ksize, stride, submanifold, stream)


def synth_kernel(desc: BasisDesc, basis: torch.Tensor, coeffs: torch.Tensor, dtype=torch.float32,
                 out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _need(basis, "basis", torch.float32)
    _need(coeffs, "coeffs", torch.float32)
    n_floats, n_coeff = basis_info(desc)
    if basis.numel() < n_floats or coeffs.numel() != n_coeff:
        raise ValueError(f"basis needs {n_floats} floats and coeffs {n_coeff} values")
    K = desc.ksize ** 3
    cin = sum(desc.in_.mult[e] * (2 * desc.in_.l[e] + 1) for e in range(desc.in_.n))
    cout = sum(desc.out.mult[e] * (2 * desc.out.l[e] + 1) for e in range(desc.out.n))
    if out is None:
        out = torch.empty((K, cout, cin), dtype=dtype, device=basis.device)
    _need(out, "W", dtype, (K, cout, cin))
    check(lib().ssconv_synth_kernel(byref(desc), _ptr(basis), _ptr(coeffs), _dtype(out), _ptr(out), _stream(stream)),
          "ssconv_synth_kernel")
    return out


def forward(feats: torch.Tensor, rb: Rulebook, W: torch.Tensor, out: Optional[torch.Tensor] = None,
            stream=None) -> torch.Tensor:
    _need(feats, "feats")
    _need(W, "W", feats.dtype)
    K, cout, cin = W.shape
    if feats.shape != (rb.n_in, cin):
        raise ValueError(f"feats must be [{rb.n_in}, {cin}]")
    if out is None:
        out = torch.empty((rb.n_out, cout), dtype=feats.dtype, device=feats.device)
    _need(out, "out", feats.dtype, (rb.n_out, cout))
    check(lib().ssconv_forward(_ptr(feats), _dtype(feats), cin, rb.handle, _ptr(W), cout, _ptr(out), _stream(stream)),
          "ssconv_forward")
    return out


def forward_noalloc(feats: torch.Tensor, rb: Rulebook, W: torch.Tensor, out: torch.Tensor, stream=None) -> torch.Tensor:
    """ssconv_forward_noalloc: forward into a caller-given out with no device allocation (scratch
    from the library's fixed per-device region)."""
    _need(feats, "feats")
    _need(W, "W", feats.dtype)
    K, cout, cin = W.shape
    if feats.shape != (rb.n_in, cin):
        raise ValueError(f"feats must be [{rb.n_in}, {cin}]")
    _need(out, "out", feats.dtype, (rb.n_out, cout))
    check(lib().ssconv_forward_noalloc(_ptr(feats), _dtype(feats), cin, rb.handle, _ptr(W), cout, _ptr(out),
                                       _stream(stream)), "ssconv_forward_noalloc")
    return out


NOALLOC_SCRATCH_BYTES = 64 << 20


def backward_workspace_size(rb: Rulebook, dtype: torch.dtype, cin: int, cout: int) -> int:
    return lib().ssconv_backward_workspace_size(rb.handle, BF16 if dtype == torch.bfloat16 else F32, cin, cout)


def backward(feats: torch.Tensor, grad_out: torch.Tensor, rb: Rulebook, W: torch.Tensor,
             desc: Optional[BasisDesc] = None, basis: Optional[torch.Tensor] = None,
             need_feats: bool = True, need_coeffs: bool = True, n_coeff: Optional[int] = None,
             workspace: Optional[torch.Tensor] = None, stream=None):
    """(grad_feats or None, grad_coeffs or None) for L = <forward(feats), grad_out>."""
    _need(feats, "feats")
    _need(grad_out, "grad_out", feats.dtype)
    _need(W, "W", feats.dtype)
    K, cout, cin = W.shape
    gf = torch.empty_like(feats) if need_feats else None
    gc = None
    if need_coeffs:
        if desc is None or basis is None:
            raise ValueError("desc and basis are required for the coefficient gradient")
        if n_coeff is None:
            n_coeff = basis_info(desc)[1]
        gc = torch.empty((n_coeff,), dtype=torch.float32, device=feats.device)
    ws_bytes = backward_workspace_size(rb, feats.dtype, cin, cout)
    if workspace is None or workspace.numel() < ws_bytes:
        workspace = torch.empty((max(ws_bytes, 256),), dtype=torch.uint8, device=feats.device)
    check(lib().ssconv_backward(_ptr(feats), _ptr(grad_out), _dtype(feats), cin, cout, rb.handle, _ptr(W),
                                byref(desc) if desc is not None else None, _ptr(basis), _ptr(gf), _ptr(gc),
                                _ptr(workspace), workspace.numel(), _stream(stream)),
          "ssconv_backward")
    return gf, gc


def gate_forward(fields: FieldList, x: torch.Tensor, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    _need(x, "x")
    f = make_fields(fields)
    C = n_channels(fields)
    if out is None:
        out = torch.empty((x.shape[0], C), dtype=x.dtype, device=x.device)
    check(lib().ssconv_gate_forward(byref(f), _ptr(x), _dtype(x), x.shape[0], _ptr(out), _stream(stream)),
          "ssconv_gate_forward")
    return out


def gate_backward(fields: FieldList, x: torch.Tensor, dy: torch.Tensor, stream=None) -> torch.Tensor:
    _need(x, "x")
    _need(dy, "dy", x.dtype)
    f = make_fields(fields)
    dx = torch.empty_like(x)
    check(lib().ssconv_gate_backward(byref(f), _ptr(x), _ptr(dy), _dtype(x), x.shape[0], _ptr(dx), _stream(stream)),
          "ssconv_gate_backward")
    return dx


NORM_EPS = 1e-5


def norm_forward(fields: FieldList, x: torch.Tensor, eps: float = NORM_EPS, out: Optional[torch.Tensor] = None,
                 stream=None) -> torch.Tensor:
    """Steerable normalisation (Eq. 11) of x [n, C] with statistics over all rows."""
    _need(x, "x")
    f = make_fields(fields)
    if x.dim() != 2 or x.shape[1] != n_channels(fields):
        raise ValueError(f"x must be [n, {n_channels(fields)}]")
    if out is None:
        out = torch.empty_like(x)
    _need(out, "out", x.dtype, tuple(x.shape))
    check(lib().ssconv_norm_forward(byref(f), _ptr(x), _dtype(x), x.shape[0], float(eps), _ptr(out),
                                    _stream(stream)), "ssconv_norm_forward")
    return out


def forward_norm(feats: torch.Tensor, rb: Rulebook, W: torch.Tensor, fields_out: FieldList, eps: float = NORM_EPS,
                 y: Optional[torch.Tensor] = None, z: Optional[torch.Tensor] = None, stream=None):
    """ssconv_forward_norm: (y, z) = (forward(feats), norm_forward(fields_out, y)), the Norm's
    statistics taken by the kernel that writes y.  z may be y (then y is overwritten)."""
    _need(feats, "feats")
    _need(W, "W", feats.dtype)
    K, cout, cin = W.shape
    if feats.shape != (rb.n_in, cin):
        raise ValueError(f"feats must be [{rb.n_in}, {cin}]")
    if cout != n_channels(fields_out):
        raise ValueError(f"W has {cout} output channels; fields_out has {n_channels(fields_out)}")
    if y is None:
        y = torch.empty((rb.n_out, cout), dtype=feats.dtype, device=feats.device)
    if z is None:
        z = torch.empty_like(y)
    _need(y, "y", feats.dtype, (rb.n_out, cout))
    _need(z, "z", feats.dtype, (rb.n_out, cout))
    f = make_fields(fields_out)
    check(lib().ssconv_forward_norm(_ptr(feats), _dtype(feats), cin, rb.handle, _ptr(W), byref(f), float(eps), _ptr(y),
                                    _ptr(z), _stream(stream)), "ssconv_forward_norm")
    return y, z


def norm_backward(fields: FieldList, x: torch.Tensor, dy: torch.Tensor, eps: float = NORM_EPS,
                  stream=None) -> torch.Tensor:
    _need(x, "x")
    _need(dy, "dy", x.dtype, tuple(x.shape))
    if x.dim() != 2 or x.shape[1] != n_channels(fields):
        raise ValueError(f"x must be [n, {n_channels(fields)}]")
    f = make_fields(fields)
    dx = torch.empty_like(x)
    check(lib().ssconv_norm_backward(byref(f), _ptr(x), _ptr(dy), _dtype(x), x.shape[0], float(eps), _ptr(dx),
                                     _stream(stream)), "ssconv_norm_backward")
    return dx


# ---- norm of a site, residual tail, checkpoints ---------------------------------------------
# A call on a few sites is over in a few microseconds, so what a field list says is looked up once and the arguments'
# checks take one comparison each where they pass.

def _on(stream):
    """Results and scratch of a call on a given stream come from that stream's memory: a block of another stream may
    still be in use there, or be handed out again there before the call has run."""
    return nullcontext() if stream is None else torch.cuda.stream(stream)


class _Table:
    """A field list: its C structure, channels, fields, checkpoint blocks (0: the library refuses the list)."""

    def __init__(self, fields):
        self.fields = fields
        self.struct = make_fields(fields)
        self.ref = byref(self.struct)
        self.C = n_channels(fields)
        self.F = sum(m for _, m in fields)
        self.blocks = int(lib().ssconv_packed_blocks(self.ref))
        self.error = "" if self.blocks else lib().ssconv_last_error().decode()
        self.gates = sum(m for l, m in fields if l > 0)
        self.full_fields = fields + (((0, self.gates),) if self.gates else ())
        self._full = None

    @property
    def full(self) -> "_Table":
        """The fields with their gates."""
        if self._full is None:
            self._full = _table(self.full_fields)
        return self._full


def _whole(v) -> int:
    i = int(v)
    if i != v or abs(i) >= 1 << 31:
        raise ValueError(f"orders and multiplicities are whole numbers of 32 bits, got {v!r}")
    return i


@lru_cache(maxsize=256)
def _table_of(fields) -> _Table:
    fields = tuple((_whole(l), _whole(m)) for l, m in fields)
    if not 1 <= len(fields) <= MAX_ENTRIES:
        raise ValueError(f"a field list has 1 to {MAX_ENTRIES} entries")
    return _Table(fields)


def _table(fields: FieldList) -> _Table:
    try:
        return _table_of(fields)
    except TypeError:                       # a list, or lists in it
        return _table_of(tuple(tuple(e) for e in fields))


def gate_fields(fields: FieldList) -> Tuple[Tuple[int, int], ...]:
    """The fields with their gate channels (one scalar per field of order > 0) as one more entry."""
    return _table(fields).full_fields


def packed_blocks(fields: FieldList) -> int:
    """Exponent bytes of a row of a checkpoint (ssconv_packed_blocks); raises for a bad list."""
    t = _table(fields)
    if t.blocks == 0:
        raise ValueError(f"bad field list {t.fields}: {t.error}")
    return t.blocks


@dataclass
class Packed:
    """An 8-bit checkpoint of rows [n, C] (ssconv_pack): int8 values [n, C] and one exponent byte per row and block of
    32 channels of an entry of ``fields``, [n, packed_blocks(fields)]."""
    fields: Tuple[Tuple[int, int], ...]
    q: torch.Tensor
    exps: torch.Tensor

    @property
    def shape(self):
        return self.q.shape

    @property
    def device(self):
        return self.q.device

    @property
    def nbytes(self) -> int:
        return self.q.numel() + self.exps.numel()

    @staticmethod
    def empty(fields: FieldList, n: int, device) -> "Packed":
        t = _table(fields)
        return Packed(t.fields, torch.empty((n, t.C), dtype=torch.int8, device=device),
                      torch.empty((n, packed_blocks(t.fields)), dtype=torch.uint8, device=device))


def _new_packed(t: _Table, n: int, like: torch.Tensor) -> Packed:
    blocks = t.blocks or packed_blocks(t.fields)
    return Packed(t.fields, like.new_empty((n, t.C), dtype=torch.int8), like.new_empty((n, blocks), dtype=torch.uint8))


def _check(t: torch.Tensor, name: str, dev: int, dtype, shape):
    """A contiguous tensor of this type and shape on the current device."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == dev and t.is_contiguous():
        return
    _need(t, name, dtype, shape)
    raise ValueError(f"{name} is on {t.device}, the current device is cuda:{dev}")


def _rows_of(x: torch.Tensor, name: str, dev: int, C: int) -> int:
    """Rows of a feature matrix of C channels."""
    if x.dim() != 2 or x.shape[1] != C:
        _need(x, name)
        raise ValueError(f"{name} must be [n, {C}], got {tuple(x.shape)}")
    n = x.shape[0]
    _dtype(x)
    _check(x, name, dev, x.dtype, (n, C))
    return n


def _check_packed(p: Packed, name: str, dev: int, t: _Table, n: int):
    if p.fields is not t.fields and _table(p.fields).fields != t.fields:
        raise ValueError(f"{name} is a checkpoint of fields {tuple(p.fields)}, not {t.fields}")
    _check(p.q, name + ".q", dev, torch.int8, (n, t.C))
    _check(p.exps, name + ".exps", dev, torch.uint8, (n, t.blocks or packed_blocks(t.fields)))


def _check_rows(x, name: str, dev: int, t: _Table, n: int, dtype) -> Rows:
    """Rows in ``dtype`` or a checkpoint of them, as the library takes them."""
    if isinstance(x, Packed):
        _check_packed(x, name, dev, t, n)
        return Rows(x.q.data_ptr(), x.exps.data_ptr())
    _check(x, name, dev, dtype, (n, t.C))
    return Rows(x.data_ptr(), None)


def _param(p: Optional[torch.Tensor], name: str, dev: int, t: _Table):
    if p is None:
        return None
    _check(p, name, dev, torch.float32, (t.F,))
    return p.data_ptr()


def _workspace(ws: Optional[torch.Tensor], need: int, dev: int, device) -> Optional[torch.Tensor]:
    if ws is None:
        return torch.empty((need,), dtype=torch.uint8, device=device) if need else None
    _check(ws, "workspace", dev, torch.uint8, (ws.numel(),))
    if ws.numel() < need:
        raise ValueError(f"workspace must hold {need} bytes, got {ws.numel()}")
    return ws


def _raw_stream(stream, dev: int) -> int:
    if stream is None:
        return torch._C._cuda_getCurrentRawStream(dev)
    if stream.device_index != dev:
        raise ValueError(f"the stream is of cuda:{stream.device_index}, the current device is cuda:{dev}")
    return stream.cuda_stream


def pack(fields: FieldList, x: torch.Tensor, stream=None) -> Packed:
    """An 8-bit checkpoint of x [n, C]."""
    t, dev = _table(fields), torch.cuda.current_device()
    n = _rows_of(x, "x", dev, t.C)
    with _on(stream):
        p = _new_packed(t, n, x)
    check(lib().ssconv_pack(t.ref, x.data_ptr(), _dtype(x), n, p.q.data_ptr(), p.exps.data_ptr(),
                            _raw_stream(stream, dev)), "ssconv_pack")
    return p


def unpack(p: Packed, dtype=torch.bfloat16, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """The values that a checkpoint stands for (exact in either type)."""
    t, dev = _table(p.fields), torch.cuda.current_device()
    n = p.q.shape[0]
    _check_packed(p, "p", dev, t, n)
    if out is None:
        with _on(stream):
            out = p.q.new_empty((n, t.C), dtype=dtype)
    _check(out, "out", dev, dtype, (n, t.C))
    check(lib().ssconv_unpack(t.ref, p.q.data_ptr(), p.exps.data_ptr(), n, _dtype(out), out.data_ptr(),
                              _raw_stream(stream, dev)), "ssconv_unpack")
    return out


def site_norm_forward(fields: FieldList, x: Union[torch.Tensor, Packed], gain: Optional[torch.Tensor] = None,
                      eps: float = NORM_EPS, out: Optional[torch.Tensor] = None, checkpoint: bool = False,
                      dtype: Optional[torch.dtype] = None, stream=None):
    """ssconv_site_norm_forward: the norm of every site of x [n, C] (or of a checkpoint; ``dtype`` is then the
    result's, bf16 unless given).  With ``checkpoint``: (y, checkpoint of x).  ``out`` may be x."""
    t, dev = _table(fields), torch.cuda.current_device()
    g = _param(gain, "gain", dev, t)
    if isinstance(x, Packed):
        if checkpoint:
            raise ValueError("x is a checkpoint already")
        n = x.q.shape[0]
        dtype = dtype or (torch.bfloat16 if out is None else out.dtype)
        r = _check_rows(x, "x", dev, t, n, None)
    else:
        n = _rows_of(x, "x", dev, t.C)
        if dtype is not None and dtype != x.dtype:
            raise TypeError(f"the result of {x.dtype} rows is {x.dtype}, not {dtype}")
        dtype = x.dtype
        r = Rows(x.data_ptr(), None)
    with _on(stream):
        if out is None:
            out = x.q.new_empty((n, t.C), dtype=dtype) if isinstance(x, Packed) else torch.empty_like(x)
        else:
            _check(out, "out", dev, dtype, (n, t.C))
        p = _new_packed(t, n, x) if checkpoint else None
    check(lib().ssconv_site_norm_forward(t.ref, byref(r), _dtype(out), n, eps, g, out.data_ptr(),
                                         p.q.data_ptr() if p else None, p.exps.data_ptr() if p else None,
                                         _raw_stream(stream, dev)), "ssconv_site_norm_forward")
    return (out, p) if checkpoint else out


def site_norm_backward(fields: FieldList, x: Union[torch.Tensor, Packed], dy: torch.Tensor,
                       gain: Optional[torch.Tensor] = None, eps: float = NORM_EPS,
                       dres: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None,
                       workspace: Optional[torch.Tensor] = None, stream=None):
    """ssconv_site_norm_backward: (gradient of x plus dres, gradient of the gain or None without one).  ``out`` may be
    dy or dres."""
    t, dev = _table(fields), torch.cuda.current_device()
    n, dtype = _rows_of(dy, "dy", dev, t.C), dy.dtype
    shape = (n, t.C)
    r = _check_rows(x, "x", dev, t, n, dtype)
    if dres is not None:
        _check(dres, "dres", dev, dtype, shape)
    g = _param(gain, "gain", dev, t)
    with _on(stream):
        if out is None:
            out = torch.empty_like(dy)
        else:
            _check(out, "out", dev, dtype, shape)
        dgain = ws = None
        if gain is not None:
            dgain = torch.empty_like(gain)
            ws = _workspace(workspace, lib().ssconv_site_norm_workspace_size(t.ref, n), dev, dy.device)
    check(lib().ssconv_site_norm_backward(t.ref, byref(r), dy.data_ptr(), None if dres is None else dres.data_ptr(),
                                          _dtype(dy), n, eps, g, out.data_ptr(),
                                          None if dgain is None else dgain.data_ptr(),
                                          None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
                                          _raw_stream(stream, dev)), "ssconv_site_norm_backward")
    return out, dgain


def residual_forward(fields: FieldList, y: torch.Tensor, h: torch.Tensor, scale: Optional[torch.Tensor] = None,
                     gain_post: Optional[torch.Tensor] = None, gain_next: Optional[torch.Tensor] = None,
                     eps: float = NORM_EPS, next_norm: bool = True, checkpoint: bool = False,
                     out: Optional[torch.Tensor] = None, stream=None):
    """ssconv_residual_forward: (h_out, x_out, checkpoint of y, checkpoint of h_out) of the convolution output y
    [n, C + G] and the residual stream h [n, C]; x_out is None without ``next_norm``, the checkpoints without
    ``checkpoint`` (and the one of h_out without ``next_norm``, whose backward alone reads it).  ``out`` may be h."""
    t, dev = _table(fields), torch.cuda.current_device()
    full = t.full
    n, dtype = _rows_of(h, "h", dev, t.C), h.dtype
    shape = (n, t.C)
    _check(y, "y", dev, dtype, (n, full.C))
    s, gp, gn = _param(scale, "scale", dev, t), _param(gain_post, "gain_post", dev, full), _param(gain_next, "gain_next", dev, t)
    if gn is not None and not next_norm:
        raise ValueError("gain_next without the next norm")
    with _on(stream):
        if out is None:
            out = torch.empty_like(h)
        else:
            _check(out, "out", dev, dtype, shape)
        x_out = torch.empty_like(h) if next_norm else None
        yp = _new_packed(full, n, h) if checkpoint else None
        hp = _new_packed(t, n, h) if checkpoint and next_norm else None
    check(lib().ssconv_residual_forward(t.ref, y.data_ptr(), h.data_ptr(), _dtype(h), n, eps, gp, s, gn, out.data_ptr(),
                                        x_out.data_ptr() if next_norm else None,
                                        yp.q.data_ptr() if yp else None, yp.exps.data_ptr() if yp else None,
                                        hp.q.data_ptr() if hp else None, hp.exps.data_ptr() if hp else None,
                                        _raw_stream(stream, dev)), "ssconv_residual_forward")
    return out, x_out, yp, hp


def residual_backward(fields: FieldList, y: Union[torch.Tensor, Packed],
                      h_out: Optional[Union[torch.Tensor, Packed]], dh: torch.Tensor,
                      dx: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                      gain_post: Optional[torch.Tensor] = None, gain_next: Optional[torch.Tensor] = None,
                      eps: float = NORM_EPS, workspace: Optional[torch.Tensor] = None, stream=None):
    """ssconv_residual_backward: (dy, gradient of h, dscale, dgain_post, dgain_next) from the gradients dh of h_out and
    dx of x_out (None without the next norm; h_out may then be None); y and h_out both as rows or both as checkpoints.  The
    gradient of a parameter that is None is None."""
    t, dev = _table(fields), torch.cuda.current_device()
    full = t.full
    n, dtype = _rows_of(dh, "dh", dev, t.C), dh.dtype
    yr = _check_rows(y, "y", dev, full, n, dtype)
    hr = Rows()
    if dx is not None:
        _check(dx, "dx", dev, dtype, (n, t.C))
        if h_out is None:
            raise ValueError("dx needs h_out")
        if isinstance(y, Packed) != isinstance(h_out, Packed):
            raise ValueError("y and h_out are rows, or both are checkpoints")
        hr = _check_rows(h_out, "h_out", dev, t, n, dtype)
    elif gain_next is not None:
        raise ValueError("gain_next without dx")
    s, gp, gn = _param(scale, "scale", dev, t), _param(gain_post, "gain_post", dev, full), _param(gain_next, "gain_next", dev, t)
    with _on(stream):
        dy = dh.new_empty((n, full.C))
        dh_in = torch.empty_like(dh)
        ds = None if s is None else torch.empty_like(scale)
        dp = None if gp is None else torch.empty_like(gain_post)
        dn = None if gn is None else torch.empty_like(gain_next)
        ws = None
        if s is not None or gp is not None or gn is not None:
            ws = _workspace(workspace, lib().ssconv_residual_workspace_size(t.ref, n), dev, dh.device)
    check(lib().ssconv_residual_backward(t.ref, byref(yr), byref(hr), dh.data_ptr(),
                                         None if dx is None else dx.data_ptr(), _dtype(dh), n, eps, gp, s, gn,
                                         dy.data_ptr(), dh_in.data_ptr(), None if dp is None else dp.data_ptr(),
                                         None if ds is None else ds.data_ptr(), None if dn is None else dn.data_ptr(),
                                         None if ws is None else ws.data_ptr(), 0 if ws is None else ws.numel(),
                                         _raw_stream(stream, dev)), "ssconv_residual_backward")
    return dy, dh_in, ds, dp, dn


def backward_packed_workspace_size(rb: Rulebook, dtype: torch.dtype, cin: int, cout: int) -> int:
    return lib().ssconv_backward_packed_workspace_size(rb.handle, BF16 if dtype == torch.bfloat16 else F32, cin, cout)


def backward_packed(feats: Packed, grad_out: torch.Tensor, rb: Rulebook, W: torch.Tensor,
                    desc: Optional[BasisDesc] = None, basis: Optional[torch.Tensor] = None, norm: bool = False,
                    gain: Optional[torch.Tensor] = None, eps: float = NORM_EPS, need_feats: bool = True,
                    need_coeffs: bool = True, n_coeff: Optional[int] = None,
                    workspace: Optional[torch.Tensor] = None, stream=None):
    """ssconv_backward_packed: ``backward`` of a convolution whose input is the checkpoint ``feats`` (``norm``: the site
    norm of it, with ``gain``)."""
    t, dev = _table(feats.fields), torch.cuda.current_device()
    _check_packed(feats, "feats", dev, t, rb.n_in)
    if W.dim() != 3 or W.shape[0] != rb.K or W.shape[2] != t.C:
        raise ValueError(f"W must be [{rb.K}, cout, {t.C}], got {tuple(W.shape)}")
    K, cout, cin = W.shape
    _check(W, "W", dev, grad_out.dtype, (K, cout, cin))
    _dtype(grad_out)
    _check(grad_out, "grad_out", dev, grad_out.dtype, (rb.n_out, cout))
    g = _param(gain, "gain", dev, t)
    if g is not None and not norm:
        raise ValueError("gain without the norm")
    coeffs = 0
    if need_coeffs:
        if desc is None or basis is None:
            raise ValueError("desc and basis are required for the coefficient gradient")
        floats, coeffs = basis_info(desc)
        if n_coeff is not None and n_coeff != coeffs:
            raise ValueError(f"the layer has {coeffs} coefficients, not {n_coeff}")
        _check(basis, "basis", dev, torch.float32, basis.shape)
        if basis.numel() < floats:
            raise ValueError(f"basis needs {floats} floats")
    with _on(stream):
        gf = torch.empty((rb.n_in, cin), dtype=grad_out.dtype, device=grad_out.device) if need_feats else None
        gc = torch.empty((coeffs,), dtype=torch.float32, device=grad_out.device) if need_coeffs else None
        ws = _workspace(workspace, backward_packed_workspace_size(rb, grad_out.dtype, cin, cout), dev, grad_out.device)
    check(lib().ssconv_backward_packed(t.ref, feats.q.data_ptr(), feats.exps.data_ptr(), int(bool(norm)), eps, g,
                                       grad_out.data_ptr(), _dtype(grad_out), cout, rb.handle, W.data_ptr(),
                                       byref(desc) if desc is not None else None, _ptr(basis), _ptr(gf), _ptr(gc),
                                       _ptr(ws), 0 if ws is None else ws.numel(), _raw_stream(stream, dev)),
          "ssconv_backward_packed")
    return gf, gc


def pool_forward(feats: torch.Tensor, rb: Rulebook, out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """2x2x2 average pooling over a rule book built with ksize 2, stride 2."""
    _need(feats, "feats")
    if feats.dim() != 2 or feats.shape[0] != rb.n_in:
        raise ValueError(f"feats must be [{rb.n_in}, C]")
    C = feats.shape[1]
    if out is None:
        out = torch.empty((rb.n_out, C), dtype=feats.dtype, device=feats.device)
    _need(out, "out", feats.dtype, (rb.n_out, C))
    check(lib().ssconv_pool_forward(_ptr(feats), _dtype(feats), C, rb.handle, _ptr(out), _stream(stream)),
          "ssconv_pool_forward")
    return out


def pool_backward(grad_out: torch.Tensor, rb: Rulebook, stream=None) -> torch.Tensor:
    _need(grad_out, "grad_out")
    if grad_out.dim() != 2 or grad_out.shape[0] != rb.n_out:
        raise ValueError(f"grad_out must be [{rb.n_out}, C]")
    C = grad_out.shape[1]
    gf = torch.empty((rb.n_in, C), dtype=grad_out.dtype, device=grad_out.device)
    check(lib().ssconv_pool_backward(_ptr(grad_out), _dtype(grad_out), C, rb.handle, _ptr(gf), _stream(stream)),
          "ssconv_pool_backward")
    return gf


def voxelize(points: torch.Tensor, feats: Optional[torch.Tensor] = None, batch: Optional[torch.Tensor] = None,
             nbatch: int = 1, origin=(0.0, 0.0, 0.0), voxel: float = 1.0, grid=64, stream=None):
    """Voxelisation with per-cell feature averaging (Sec. 4.1).  Returns (coords [m, 4] int32,
    averaged feats [m, C] fp32 or None, point_row [n] int32); with a batch tensor, nbatch
    must cover its indices."""
    _need(points, "points", torch.float32)
    if points.dim() != 2 or points.shape[1] != 3:
        raise ValueError("points must be [n, 3]")
    n = points.shape[0]
    C = 0
    if feats is not None:
        _need(feats, "feats", torch.float32)
        if feats.dim() != 2 or feats.shape[0] != n:
            raise ValueError(f"feats must be [{n}, C]")
        C = feats.shape[1]
    if batch is not None:
        _need(batch, "batch", torch.int32, (n,))
    g = (c_int * 3)(*([int(grid)] * 3 if np.isscalar(grid) else [int(v) for v in grid]))
    o = (c_float * 3)(*[float(v) for v in origin])
    coords = torch.empty((n, 4), dtype=torch.int32, device=points.device)
    fo = torch.empty((n, C), dtype=torch.float32, device=points.device) if C else None
    rows = torch.empty((n,), dtype=torch.int32, device=points.device)
    m = c_int64()
    check(lib().ssconv_voxelize(_ptr(points), _ptr(batch), _ptr(feats), n, C, o, float(voxel), g, int(nbatch),
                                _ptr(coords), _ptr(fo), _ptr(rows), byref(m), _stream(stream)), "ssconv_voxelize")
    k = m.value
    return coords[:k], (fo[:k] if fo is not None else None), rows


def wigner_d(l: int, rot) -> np.ndarray:
    """D^l(rot) of the real harmonic basis (host computation)."""
    d = 2 * int(l) + 1
    r = (ctypes.c_double * 9)(*[float(v) for v in np.asarray(rot, np.float64).reshape(9)])
    out = (ctypes.c_double * (d * d))()
    check(lib().ssconv_wigner_d(int(l), r, out), "ssconv_wigner_d")
    return np.array(out[:], np.float64).reshape(d, d)


def steer(coords: torch.Tensor, feats: torch.Tensor, fields: FieldList, rot, trans, nbatch: int = 1,
          origin=(0.0, 0.0, 0.0), voxel: float = 1.0, grid=64, stream=None):
    """Feature-Steering (Sec. 4.1) by p -> rot p + trans.  Returns (coords' [m, 4] int32,
    feats' [m, C] fp32, site_row [n] int32)."""
    _need(coords, "coords", torch.int32)
    _need(feats, "feats", torch.float32)
    n = coords.shape[0]
    C = n_channels(fields)
    if coords.dim() != 2 or coords.shape[1] != 4 or tuple(feats.shape) != (n, C):
        raise ValueError(f"coords must be [n, 4] and feats [n, {C}]")
    f = make_fields(fields)
    r = (ctypes.c_double * 9)(*[float(v) for v in np.asarray(rot, np.float64).reshape(9)])
    t = (ctypes.c_double * 3)(*[float(v) for v in np.asarray(trans, np.float64).reshape(3)])
    g = (c_int * 3)(*([int(grid)] * 3 if np.isscalar(grid) else [int(v) for v in grid]))
    o = (c_float * 3)(*[float(v) for v in origin])
    co = torch.empty((n, 4), dtype=torch.int32, device=coords.device)
    fo = torch.empty((n, C), dtype=torch.float32, device=coords.device)
    rows = torch.empty((n,), dtype=torch.int32, device=coords.device)
    m = c_int64()
    check(lib().ssconv_steer(_ptr(coords), _ptr(feats), n, byref(f), r, t, o, float(voxel), g, int(nbatch), _ptr(co),
                             _ptr(fo), _ptr(rows), byref(m), _stream(stream)), "ssconv_steer")
    k = m.value
    return co[:k], fo[:k], rows


def _interp_args(rb, points, batch, C):
    _need(points, "points", torch.float32)
    if points.dim() != 2 or points.shape[1] != 3:
        raise ValueError("points must be [m, 3]")
    if batch is not None:
        _need(batch, "batch", torch.int32, (points.shape[0],))
    if C < 1:
        raise ValueError("channels must be positive")


def interpolate(rb: Rulebook, feats: torch.Tensor, points: torch.Tensor, batch: Optional[torch.Tensor] = None,
                origin=(0.0, 0.0, 0.0), voxel: float = 1.0, stream=None) -> torch.Tensor:
    """Tensor-to-Point (Sec. 4.1): trilinear interpolation of the sites' features at points."""
    _need(feats, "feats", torch.float32)
    if feats.dim() != 2 or feats.shape[0] != rb.n_in:
        raise ValueError(f"feats must be [{rb.n_in}, C]")
    C = feats.shape[1]
    _interp_args(rb, points, batch, C)
    out = torch.empty((points.shape[0], C), dtype=torch.float32, device=points.device)
    o = (c_float * 3)(*[float(v) for v in origin])
    check(lib().ssconv_interpolate(rb.handle, _ptr(feats), C, _ptr(points), _ptr(batch), points.shape[0], o,
                                   float(voxel), _ptr(out), _stream(stream)), "ssconv_interpolate")
    return out


def interpolate_backward(rb: Rulebook, grad: torch.Tensor, points: torch.Tensor, batch: Optional[torch.Tensor] = None,
                         origin=(0.0, 0.0, 0.0), voxel: float = 1.0, stream=None) -> torch.Tensor:
    _need(grad, "grad", torch.float32)
    if grad.dim() != 2 or grad.shape[0] != points.shape[0]:
        raise ValueError("grad must be [m, C]")
    C = grad.shape[1]
    _interp_args(rb, points, batch, C)
    gf = torch.empty((rb.n_in, C), dtype=torch.float32, device=points.device)
    o = (c_float * 3)(*[float(v) for v in origin])
    check(lib().ssconv_interpolate_backward(rb.handle, _ptr(grad), C, _ptr(points), _ptr(batch), points.shape[0], o,
                                            float(voxel), _ptr(gf), _stream(stream)), "ssconv_interpolate_backward")
    return gf


def debug_set(option: int, value: int) -> None:
    check(lib().ssconv_debug_set(int(option), int(value)), "ssconv_debug_set")


def empty_cache() -> None:
    """Waits for and releases the library's cached free device blocks."""
    check(lib().ssconv_empty_cache(), "ssconv_empty_cache")


def cached_bytes() -> int:
    """Bytes held in the library's cached free device blocks."""
    return int(lib().ssconv_cached_bytes())


def debug_kernel_ms() -> Tuple[int, float]:
    """(launches, total ms) of the gather-GEMM kernels timed on this thread since
    debug_set(4, 1); waits for the last of them."""
    n, ms = c_int64(), c_float()
    check(lib().ssconv_debug_kernel_ms(byref(n), byref(ms)), "ssconv_debug_kernel_ms")
    return int(n.value), float(ms.value)
