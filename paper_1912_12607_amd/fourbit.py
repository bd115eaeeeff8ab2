"""Token operators in microscaled 4-bit codes over the C ABI: linear layers (for training and for serving), a paged cache of keys and values, and attention over it.

Plumbing only, as in ``tokens``, whose operators these are in half the memory: blocks of 32 values along the axis that a product sums over share a power of two.
NaN and infinities make their block, and what is computed from it, NaN.

    layer = ServedLinear4.of(weight, bias)              # codes and scales, laid out once
    cache = PagedCache4.empty(pages, page_size, heads, dim, device)
    cache.write(k, v, slots)                            # quantised on the way in
    o = cache.attend(q, starts, lengths, table)         # the new tokens of each request over its pages
    y = linear4(x, weight, bias, seed=7)                # differentiable; TokenLinear4 is the module
"""
from __future__ import annotations

import functools

import torch

from . import binding as B
from .tokens import PagedCache, TokenLinear, _call, _rows, _tangent, _transformed, _type, _vector


def _blocks(n: int) -> int:
    return (n + 31) // 32


def _panels(n: int) -> int:
    return (n + 255) // 256


@functools.lru_cache(maxsize=1024)
def _plan(M: int, K: int, N: int, kind: int, wkind: int):
    """What calls of these sizes have in common: the descriptor, scratch bytes of its directions (forward, backward, served), and where the backward pass's codes
    and scales (of x and W by columns) lie in one piece of memory, and its size."""
    desc = B.LinearDesc(M, K, N, kind, wkind)
    need = tuple(B.lib.int8t_mx4_linear_workspace_bytes(desc, i) for i in range(3))
    at, places = 0, []
    for n in (K * 16 * _blocks(M), K * 8 * _panels(M), K * 16 * _blocks(N), K * 8 * _panels(N)):
        places.append(at)
        at += (n + 255) & ~255
    return desc, need, tuple(places), at


class ServedLinear4:
    """A linear layer in use: weights as codes with a scale for each 32 inputs of an output channel, laid out once; each token's blocks get their scales when it
    arrives.  y = x W^T + b in x's type; no gradients.

    codes: (out, 16 * blocks) uint8, blocks = in / 32 rounded up: two codes to a byte, the first in the low half, zero beyond in
    scales: (out, blocks, or more columns that are not used) uint8: 2^(byte - 127)"""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, in_features: int, bias: torch.Tensor | None = None):
        n, blocks, panels = int(in_features), _blocks(in_features), _panels(in_features)
        if codes.dtype is not torch.uint8 or codes.dim() != 2 or codes.shape[1] != 16 * blocks or not codes.is_contiguous() or not codes.is_cuda:
            raise RuntimeError(f"codes: contiguous uint8 (out, {16 * blocks}) on the device, not {tuple(codes.shape)} of {codes.dtype}")
        out, index = codes.shape[0], codes.get_device()
        if scales.dtype is not torch.uint8 or scales.dim() != 2 or scales.shape[0] != out or scales.shape[1] < blocks or scales.get_device() != index:
            raise RuntimeError(f"scales: uint8 ({out}, {blocks}) on {codes.device}, not {tuple(scales.shape)} of {scales.dtype} on {scales.device}")
        whole = torch.zeros(out, 8 * panels, dtype=torch.uint8, device=codes.device)
        whole[:, :blocks] = scales[:, :blocks]
        self._set(codes, whole.view(out, panels, 8).transpose(0, 1).contiguous(), n, bias)

    def _set(self, codes, panels, n, bias):
        self.in_features, self.out_features = n, codes.shape[0]
        self._index = codes.get_device()
        self._tensors = codes, panels, _vector(bias, codes.shape[0], "bias", self._index)
        self._b = B.Mx4LinearBuffers(wq=codes.data_ptr(), sw=panels.data_ptr(), bias=None if self.bias is None else self.bias.data_ptr(), y_pitch=self.out_features)

    # (not to be replaced: their addresses are taken once)
    codes = property(lambda self: self._tensors[0])
    bias = property(lambda self: self._tensors[2])

    @property
    def scales(self) -> torch.Tensor:
        """(out, blocks), a copy."""
        return self._tensors[1].transpose(0, 1).reshape(self.out_features, -1)[:, :_blocks(self.in_features)].contiguous()

    @classmethod
    def of(cls, weight: torch.Tensor, bias: torch.Tensor | None = None) -> "ServedLinear4":
        """From floating weights (out, in): nearest codes."""
        if weight.dim() != 2:
            raise RuntimeError(f"weight of {weight.dim()} dimensions")
        kind = _type(weight, "weight")
        N, K = weight.shape
        w, pitch = _rows(weight.detach(), K)
        codes = torch.empty(N, 16 * _blocks(K), dtype=torch.uint8, device=w.device)
        panels = torch.empty(_panels(K), N, 8, dtype=torch.uint8, device=w.device)
        _call(w.get_device(), B.lib.int8t_mx4_quantize, w.data_ptr(), kind, N, K, pitch, B.ROUND_NEAREST_EVEN, 0, codes.data_ptr(), panels.data_ptr(), None, None, None, None, 0)
        layer = cls.__new__(cls)
        layer._set(codes, panels, K, bias)
        return layer

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        kind = B.DTYPES.get(x.dtype)
        shape = x.shape
        if kind is None or x.get_device() != self._index or not shape or shape[-1] != self.in_features:
            _type(x, "x")
            raise RuntimeError(f"input of {tuple(shape)} on {x.device} in a layer of {self.in_features} on {self.codes.device}")
        y = x.new_empty(shape[:-1] + (self.out_features,))
        if y.numel() == 0:
            return y
        rows, pitch = _rows(x, self.in_features)
        desc, (_, _, need), _, _ = _plan(rows.shape[0], self.in_features, self.out_features, kind, kind)
        b = B.Mx4LinearBuffers.from_buffer_copy(self._b)
        b.x, b.x_pitch, b.y = rows.data_ptr(), pitch, y.data_ptr()
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)
            b.ws, b.ws_bytes = ws.data_ptr(), need
        _call(self._index, B.lib.int8t_mx4_linear_fwd, desc, b)
        return y


def _linear4(x, w, bias, want_x=False, want_w=False, want_b=False):
    """(y, the plan, what the gradients that are wanted read: codes and scales of x and W by columns, in one piece of memory, or None)."""
    kind, wkind = _type(x, "x"), _type(w, "weight")
    shape = x.shape
    if w.dim() != 2 or not shape or shape[-1] != w.shape[1] or w.device != x.device:
        raise RuntimeError(f"input of {tuple(shape)} on {x.device}, weight of {tuple(w.shape)} on {w.device}")
    N, K = w.shape
    index, dev = x.get_device(), x.device
    bias = _vector(bias, N, "bias", index)
    (rows, pitch), (wr, w_pitch) = _rows(x, K), _rows(w, K)
    M = rows.shape[0]
    y = x.new_empty(shape[:-1] + (N,))
    plan = desc, (need, later, _), places, size = _plan(M, K, N, kind, wkind)
    kept = None
    if M:
        b = B.Mx4LinearBuffers()
        if (want_x or want_w or want_b) and not later:
            raise RuntimeError(f"{M} tokens, {K} inputs, {N} outputs: a backward pass of that size is not served")
        if want_x or want_w:
            kept = torch.empty(size, dtype=torch.uint8, device=dev)
            at = kept.data_ptr()
            if want_w:
                b.xt, b.sxt = at, at + places[1]
            if want_x:
                b.wt, b.swt = at + places[2], at + places[3]
        b.x, b.x_pitch, b.w, b.w_pitch, b.y, b.y_pitch = rows.data_ptr(), pitch, wr.data_ptr(), w_pitch, y.data_ptr(), N
        if bias is not None:
            b.bias = bias.data_ptr()
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        b.ws, b.ws_bytes = ws.data_ptr(), need
        _call(index, B.lib.int8t_mx4_linear_fwd, desc, b)
    return y, plan, kept


class _Linear4Fn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, seed):
        y, (ctx.desc, (_, ctx.need, _), ctx.places, _), kept = _linear4(x, w, bias, *ctx.needs_input_grad[:3])
        ctx.save_for_backward(*(() if kept is None else (kept,)))
        ctx.seed, ctx.x_shape, ctx.w_dtype = seed, x.shape, w.dtype
        return y

    @staticmethod
    def backward(ctx, dy):
        if torch.is_grad_enabled():
            raise RuntimeError("linear4() is differentiable once")
        if _transformed() and _tangent(dy):
            raise RuntimeError("linear4() has no forward mode, its gradient neither")
        want_x, want_w, want_b = ctx.needs_input_grad[:3]
        desc, dev = ctx.desc, dy.device
        M, K, N = desc.M, desc.K, desc.N
        dx = dy.new_empty(ctx.x_shape) if want_x else None
        if M == 0:
            return (dx, torch.zeros(N, K, dtype=ctx.w_dtype, device=dev) if want_w else None,
                    torch.zeros(N, dtype=torch.float32, device=dev) if want_b else None, None)
        g, pitch = _rows(dy, N)
        b = B.Mx4LinearBuffers()
        dw = db = None
        if want_x or want_w:
            kept, = ctx.saved_tensors
            at, places = kept.data_ptr(), ctx.places
            b.xt, b.sxt, b.wt, b.swt = at, at + places[1], at + places[2], at + places[3]
        b.dy, b.dy_pitch = g.data_ptr(), pitch
        if want_x:
            b.dx = dx.data_ptr()
        if want_w:
            dw = torch.empty(N, K, dtype=ctx.w_dtype, device=dev)
            b.dw = dw.data_ptr()
        if want_b:
            db = torch.empty(N, dtype=torch.float32, device=dev)
            b.db = db.data_ptr()
        ws = torch.empty(ctx.need, dtype=torch.uint8, device=dev)
        b.ws, b.ws_bytes = ws.data_ptr(), ctx.need
        _call(dy.get_device(), B.lib.int8t_mx4_linear_bwd, desc, b, ctx.seed)
        return dx, dw, db, None


def linear4(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, seed: int = 0) -> torch.Tensor:
    """x W^T + b, every product in microscaled 4-bit codes with blocks along its summed axis, differentiable (once): the gradients' codes are rounded
    stochastically with draws of `seed`.  Where no graph records it is the forward pass alone.  x (.., in) and weight (out, in) fp32, bf16 or fp16; bias fp32.  A pass that is captured into a CUDA graph takes leaves of which no
    eager autograd graph lives any more (torch would join the streams of both, and ends the process)."""
    # (what no graph records keeps nothing: a Function's needs_input_grad goes by the leaves alone)
    if not _transformed() and not (torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or (bias is not None and bias.requires_grad))):
        return _linear4(x, weight, bias)[0]
    return _Linear4Fn.apply(x, weight, bias, int(seed) & 0xFFFFFFFFFFFFFFFF)


class TokenLinear4(TokenLinear):
    """`TokenLinear` through linear4()."""

    def forward(self, x):
        if torch.is_grad_enabled():
            self._seed += 1
        return linear4(x, self.weight, self.bias, self._seed)

    def served(self) -> ServedLinear4:
        """The layer with its present weights, for use without gradients."""
        return ServedLinear4.of(self.weight, self.bias if self.bias is None else self.bias.detach())


class PagedCache4(PagedCache):
    """`PagedCache` in microscaled 4-bit codes, blocks along a head's dims: 4.25 bits a value.

    kq, vq: (pages, heads, page_size, 16 * blocks) uint8;  ks, vs: (pages, heads, page_size, blocks) uint8;  blocks = dim / 32 rounded up"""

    _calls = B.lib.int8t_mx4_cache_write, B.lib.int8t_mx4_cache_read, B.lib.int8t_mx4_cache_attend_workspace_bytes, B.lib.int8t_mx4_cache_attend

    def __init__(self, kq, ks, vq, vs, dim: int):
        blocks = _blocks(dim)
        if kq.dim() != 4 or kq.shape[3] != 16 * blocks or kq.shape != vq.shape or ks.shape != kq.shape[:3] + (blocks,) or vs.shape != ks.shape:
            raise RuntimeError(f"cache of codes {tuple(kq.shape)}, {tuple(vq.shape)} and scales {tuple(ks.shape)}, {tuple(vs.shape)} for heads of {dim}")
        for t, name in ((kq, "kq"), (vq, "vq"), (ks, "ks"), (vs, "vs")):
            if t.dtype is not torch.uint8 or not t.is_cuda or not t.is_contiguous() or t.device != kq.device:
                raise RuntimeError(f"{name}: contiguous uint8 on {kq.device}")
        self._keep(B.Mx4Cache, kq, ks, vq, vs, int(dim))

    @classmethod
    def empty(cls, pages: int, page_size: int, heads: int, dim: int, device="cuda:0") -> "PagedCache4":
        q = [torch.zeros(pages, heads, page_size, 16 * _blocks(dim), dtype=torch.uint8, device=device) for _ in range(2)]
        s = [torch.zeros(pages, heads, page_size, _blocks(dim), dtype=torch.uint8, device=device) for _ in range(2)]
        return cls(q[0], s[0], q[1], s[1], dim)
