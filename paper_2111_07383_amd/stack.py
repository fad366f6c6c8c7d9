"""A stack of SS-Conv layers with the gated nonlinearity between them (Sec. 3.2-3.3), the
paper's downsampling block (stride-1 SS-Conv, Norm, gate, average pooling), and a residual trunk of
stride-1 SS-Convs between the norms of a site.

Every step calls the C ABI through ``binding``; this module only sequences the
calls and keeps what the backward pass needs.  A layer object provides
``fields_in``, ``fields_out`` (gate channels included when ``gated``),
``ksize``, ``stride``, ``submanifold``, ``shells``, ``eps``, ``jmax``, ``gated``.
"""
from dataclasses import dataclass, field
from typing import List, Optional

import torch

from . import binding as B


@dataclass
class LayerState:
    layer: object
    desc: object
    basis: torch.Tensor          # fp32 device basis of ssconv_basis_build
    coeffs: torch.Tensor         # fp32 device coefficients
    n_coeff: int
    grid: int                    # input grid extent
    rb: Optional[B.Rulebook] = None
    W: Optional[torch.Tensor] = None
    x: Optional[torch.Tensor] = None   # layer input features, or their checkpoint (B.Packed)
    y: Optional[torch.Tensor] = None   # convolution output (before the gate), or its checkpoint


def regular_fields(layer):
    """Output fields without the appended gate channels."""
    return tuple(layer.fields_out[:-1]) if layer.gated else tuple(layer.fields_out)


@dataclass
class Stack:
    """``checkpoint``: the forward keeps every layer's input and convolution output as 8-bit checkpoints
    (their values are within 1/127 of the largest of 32 channels), and the gradients are taken at those; layers then
    have at most 1024 channels."""
    layers: List[LayerState] = field(default_factory=list)
    dtype: torch.dtype = torch.float32
    checkpoint: bool = False

    @staticmethod
    def create(layer_specs, coeffs_list, grid: int, device, dtype=torch.float32, checkpoint: bool = False) -> "Stack":
        st = Stack(dtype=dtype, checkpoint=checkpoint)
        g = grid
        for spec, w in zip(layer_specs, coeffs_list):
            desc = B.layer_desc(spec)
            basis = torch.from_numpy(B.basis_build(desc)).to(device)
            n_coeff = B.basis_info(desc)[1]
            c = torch.as_tensor(w, dtype=torch.float32).to(device)
            if c.numel() != n_coeff:
                raise ValueError(f"layer expects {n_coeff} coefficients, got {c.numel()}")
            st.layers.append(LayerState(spec, desc, basis, c, n_coeff, g))
            g = -(-g // spec.stride)
        return st

    def forward(self, coords: torch.Tensor, feats: torch.Tensor, overlap: bool = True):
        """Returns (output coords, output features); rule books are rebuilt every call.

        Rule books and kernels depend on coordinates and coefficients only (a generated output set
        comes from the rule book itself), so with ``overlap`` they are prepared on a side stream
        one layer ahead: the rule-book build of layer n+1, whose host synchronisation waits on
        the side stream only, is queued while layer n's convolution runs on the caller's stream
        (measured on the five-layer stack: 5.85 -> 5.76 ms per step; a host thread running the
        builds further ahead was slower, 6.3 ms)."""
        main = torch.cuda.current_stream()
        side = self._side() if overlap else main
        side.wait_stream(main)          # the caller's coordinates, and last call's uses of the rule books
        for L in self.layers:
            if L.rb is not None:
                L.rb.close()
                L.rb = None
        with torch.cuda.stream(side):
            self._prepare(0, coords)
        h, c = feats, coords
        for i, L in enumerate(self.layers):
            s = L.layer
            main.wait_stream(side)
            if side is not main:
                L.W.record_stream(main)
            y = B.forward(h, L.rb, L.W)
            L.x = B.pack(s.fields_in, h) if self.checkpoint else h
            L.y = y
            if self.checkpoint:
                L.y = B.pack(s.fields_out, y) if s.gated else None
            h = B.gate_forward(regular_fields(s), y) if s.gated else y
            if not s.submanifold:
                with torch.cuda.stream(side):
                    c = L.rb.out_coords()
                if side is not main:
                    c.record_stream(main)
            if i + 1 < len(self.layers):
                with torch.cuda.stream(side):
                    self._prepare(i + 1, c)
        return c, h

    def _side(self) -> torch.cuda.Stream:
        if getattr(self, "_side_stream", None) is None:
            self._side_stream = torch.cuda.Stream()   # default priority
        return self._side_stream

    def _prepare(self, i: int, coords: torch.Tensor):
        """Kernel and rule book of layer i on the current stream (a generated output set's build
        synchronises it; a submanifold build is settled by the first call that needs its counts)."""
        L = self.layers[i]
        s = L.layer
        L.W = B.synth_kernel(L.desc, L.basis, L.coeffs, self.dtype)
        L.rb = B.Rulebook(coords, L.grid, s.ksize, s.stride, s.submanifold, asynchronous=True)

    def backward(self, grad: torch.Tensor, need_input_grad: bool = True):
        """Returns (grad of the stack input or None, [grad_coeffs per layer])."""
        g = grad
        gcs = [None] * len(self.layers)
        for idx in range(len(self.layers) - 1, -1, -1):
            L = self.layers[idx]
            s = L.layer
            if s.gated:
                y = B.unpack(L.y, self.dtype) if self.checkpoint else L.y
                g = B.gate_backward(regular_fields(s), y, g)
            back = B.backward_packed if self.checkpoint else B.backward
            gf, gc = back(L.x, g, L.rb, L.W, L.desc, L.basis, need_feats=(idx > 0 or need_input_grad),
                          need_coeffs=True, n_coeff=L.n_coeff)
            gcs[idx] = gc
            g = gf
        return g, gcs

    def close(self):
        if getattr(self, "_side_stream", None) is not None:
            self._side_stream.wait_stream(torch.cuda.current_stream())
        for L in self.layers:
            if L.rb is not None:
                L.rb.close()
                L.rb = None


@dataclass
class DownBlock:
    """The paper's downsampling block: a stride-1 submanifold SS-Conv, steerable Norm (Eq. 11)
    over every output field (gate channels included), the gated nonlinearity (Eq. 12), then
    2x2x2 average pooling (the footnote of Sec. 3.1).  The convolution and its Norm are one call
    (``forward_norm``: in fp32 the kernel that writes the convolution output also sums its statistics).
    Rule books are rebuilt every call."""
    state: LayerState
    dtype: torch.dtype = torch.float32
    norm_eps: float = B.NORM_EPS
    pool_rb: Optional[B.Rulebook] = None
    z: Optional[torch.Tensor] = None     # normalised convolution output (input of the gate)

    @staticmethod
    def create(layer_spec, coeffs, grid: int, device, dtype=torch.float32) -> "DownBlock":
        if layer_spec.stride != 1 or not layer_spec.submanifold:
            raise ValueError("the block's convolution is a stride-1 submanifold SS-Conv")
        st = Stack.create([layer_spec], [coeffs], grid, device, dtype)
        return DownBlock(st.layers[0], dtype)

    def forward(self, coords: torch.Tensor, feats: torch.Tensor, overlap: bool = True):
        """Returns (pooled coords, pooled features).  The pooling rule book depends on the
        coordinates only: with ``overlap`` it is built on a side stream after the convolution,
        Norm and gate are queued, so its host synchronisations overlap them."""
        L, s = self.state, self.state.layer
        main = torch.cuda.current_stream()
        side = self._side() if overlap else main
        side.wait_stream(main)
        for rb in (L.rb, self.pool_rb):
            if rb is not None:
                rb.close()
        L.W = B.synth_kernel(L.desc, L.basis, L.coeffs, self.dtype)
        L.rb = B.Rulebook(coords, L.grid, s.ksize, 1, True, asynchronous=True)
        L.x = feats
        L.y, self.z = B.forward_norm(feats, L.rb, L.W, s.fields_out, self.norm_eps)
        h = B.gate_forward(regular_fields(s), self.z) if s.gated else self.z
        with torch.cuda.stream(side):
            self.pool_rb = B.Rulebook(coords, L.grid, 2, 2, False)
            pc = self.pool_rb.out_coords()
        main.wait_stream(side)
        if side is not main:
            pc.record_stream(main)
        return pc, B.pool_forward(h, self.pool_rb)

    def _side(self) -> torch.cuda.Stream:
        if getattr(self, "_side_stream", None) is None:
            self._side_stream = torch.cuda.Stream()   # default priority
        return self._side_stream

    def backward(self, grad: torch.Tensor, need_input_grad: bool = True):
        """Returns (grad of the block input or None, grad_coeffs)."""
        L, s = self.state, self.state.layer
        g = B.pool_backward(grad, self.pool_rb)
        if s.gated:
            g = B.gate_backward(regular_fields(s), self.z, g)
        g = B.norm_backward(s.fields_out, L.y, g, self.norm_eps)
        return B.backward(L.x, g, L.rb, L.W, L.desc, L.basis, need_feats=need_input_grad, need_coeffs=True,
                          n_coeff=L.n_coeff)

    def close(self):
        if getattr(self, "_side_stream", None) is not None:
            self._side_stream.wait_stream(torch.cuda.current_stream())
        for rb in (self.state.rb, self.pool_rb):
            if rb is not None:
                rb.close()
        self.state.rb = self.pool_rb = None


@dataclass
class ResidualStack:
    """A residual trunk on one site set: block i takes the residual stream h to

        h + scale_i * gate(norm(conv_i(norm(h))))

    with the norm of a site before the convolution (gain ``gain_pre[i]``) and behind it (``gain_post[i]``, the gate
    channels included), the gated nonlinearity (Eq. 12) and a scale per field.  The convolutions are stride-1
    submanifold and gated, and keep the fields of the stream.  The tail of a block and the norm in front of the next
    are one call (``residual_forward``).

    ``checkpoint``: the forward keeps 8-bit checkpoints of each block's residual stream and convolution output and
    nothing else of its activations; the backward takes the norms again at those (a 208-channel block in bf16 keeps
    0.48 instead of 1.3 KB a site)."""
    blocks: List[LayerState] = field(default_factory=list)
    scale: List[torch.Tensor] = field(default_factory=list)       # fp32 [fields]
    gain_pre: List[torch.Tensor] = field(default_factory=list)    # fp32 [fields]
    gain_post: List[torch.Tensor] = field(default_factory=list)   # fp32 [fields + gates]
    dtype: torch.dtype = torch.float32
    eps: float = B.NORM_EPS
    checkpoint: bool = False
    h: list = field(default_factory=list)        # the stream in front of each block (rows or checkpoints)
    rulebooks: dict = field(default_factory=dict)  # by kernel size

    @staticmethod
    def create(layer_specs, coeffs_list, grid: int, device, dtype=torch.float32, scale: float = 1.0,
               eps: float = B.NORM_EPS, checkpoint: bool = False) -> "ResidualStack":
        """Gains start at one, residual scales at ``scale``."""
        specs = list(layer_specs)
        for s in specs:
            if s.stride != 1 or not s.submanifold or not s.gated:
                raise ValueError("a residual block's convolution is a gated stride-1 submanifold SS-Conv")
            if tuple(s.fields_in) != tuple(specs[0].fields_in) or tuple(s.fields_out) != B.gate_fields(s.fields_in):
                raise ValueError("a residual block keeps the fields of the stream (and adds their gate channels)")
        st = Stack.create(specs, coeffs_list, grid, device, dtype)
        r = ResidualStack(blocks=st.layers, dtype=dtype, eps=eps, checkpoint=checkpoint)
        for s in specs:
            n, full = (sum(m for _, m in f) for f in (s.fields_in, s.fields_out))
            r.scale.append(torch.full((n,), float(scale), device=device))
            r.gain_pre.append(torch.ones((n,), device=device))
            r.gain_post.append(torch.ones((full,), device=device))
        return r

    def forward(self, coords: torch.Tensor, feats: torch.Tensor) -> torch.Tensor:
        """Returns the residual stream behind the last block (rows as ``feats``); one rule book per kernel size is
        built per call."""
        self.close()
        h, self.h = feats, []
        if not self.blocks:
            return h
        fields = tuple(self.blocks[0].layer.fields_in)
        for L in self.blocks:
            if L.layer.ksize not in self.rulebooks:
                self.rulebooks[L.layer.ksize] = B.Rulebook(coords, L.grid, L.layer.ksize, 1, True, asynchronous=True)
        if self.checkpoint:
            x, kept = B.site_norm_forward(fields, h, self.gain_pre[0], self.eps, checkpoint=True)
        else:
            x, kept = B.site_norm_forward(fields, h, self.gain_pre[0], self.eps), h
        for i, L in enumerate(self.blocks):
            last = i + 1 == len(self.blocks)
            self.h.append(kept)
            L.rb = self.rulebooks[L.layer.ksize]
            L.W = B.synth_kernel(L.desc, L.basis, L.coeffs, self.dtype)
            y = B.forward(x, L.rb, L.W)
            L.x = None if self.checkpoint else x
            h, x, yk, hk = B.residual_forward(fields, y, h, self.scale[i], self.gain_post[i],
                                              None if last else self.gain_pre[i + 1], self.eps, next_norm=not last,
                                              checkpoint=self.checkpoint)
            L.y, kept = (yk, hk) if self.checkpoint else (y, h)
        return h

    def backward(self, grad: torch.Tensor):
        """(gradient of the input features, {"coeffs", "scale", "gain_pre", "gain_post": gradients per block})."""
        n = len(self.blocks)
        out = {k: [None] * n for k in ("coeffs", "scale", "gain_pre", "gain_post")}
        if n == 0:
            return grad, out
        fields = tuple(self.blocks[0].layer.fields_in)
        dh, dx = grad, None
        for i in range(n - 1, -1, -1):
            L, last = self.blocks[i], i + 1 == n
            dy, dh, out["scale"][i], out["gain_post"][i], dnext = B.residual_backward(
                fields, L.y, None if last else self.h[i + 1], dh, dx, self.scale[i], self.gain_post[i],
                None if last else self.gain_pre[i + 1], self.eps)
            if not last:
                out["gain_pre"][i + 1] = dnext
            if self.checkpoint:
                dx, out["coeffs"][i] = B.backward_packed(self.h[i], dy, L.rb, L.W, L.desc, L.basis, norm=True,
                                                         gain=self.gain_pre[i], eps=self.eps)
            else:
                dx, out["coeffs"][i] = B.backward(L.x, dy, L.rb, L.W, L.desc, L.basis, n_coeff=L.n_coeff)
        dfeats, out["gain_pre"][0] = B.site_norm_backward(fields, self.h[0], dx, self.gain_pre[0], self.eps, dres=dh)
        return dfeats, out

    def close(self):
        for rb in self.rulebooks.values():
            rb.close()
        self.rulebooks = {}
        for L in self.blocks:
            L.rb = None
