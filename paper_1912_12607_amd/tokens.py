"""Token operators over the C ABI: linear layers with a scale for each token and output channel (for training and for serving), a
paged cache of keys and values in 8 bits, and attention of new tokens over it.

Plumbing only, as in ``autograd``: every arithmetic step is one of the library's entry points; torch supplies device memory, the current
stream and the autograd graph.  CUDA(ROCm) tensors in fp32, bf16 or fp16.  NaN and infinities make what is computed from their token, channel or
cached row NaN.

    layer = ServedLinear.of(weight, bias)               # codes and scales, laid out once
    cache = PagedCache.empty(pages, page_size, heads, dim, device)
    cache.write(k, v, slots)                            # quantised on the way in
    o = cache.attend(q, starts, lengths, table)         # the new tokens of each request over its pages
    y = linear(x, weight, bias, seed=7)                 # differentiable; TokenLinear is the module
"""
from __future__ import annotations

import functools
import zlib

import torch

from . import binding as B


def _pad16(n: int) -> int:
    return (n + 15) & ~15


def _type(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise RuntimeError(f"{name} is not a device tensor")
    if t.dtype not in B.DTYPES:
        raise TypeError(f"{name} is {t.dtype}: float32, bfloat16 or float16")
    return B.DTYPES[t.dtype]


_forward_ad = torch.autograd.forward_ad
_functorch_active = getattr(torch._C, "_are_functorch_transforms_active", lambda: False)


def _transformed() -> bool:
    """Whether a call may see tensors that have tangents (a level of forward-mode differentiation), or that a transformation stands behind."""
    return getattr(_forward_ad, "_current_level", -1) >= 0 or _functorch_active()


def _tangent(t: torch.Tensor) -> bool:
    """Whether t has a tangent at the present level of forward-mode differentiation."""
    return _forward_ad.unpack_dual(t).tangent is not None


def _rows(t: torch.Tensor, cols: int):
    """(t as rows of `cols` contiguous values, elements between rows); a copy where its strides do not allow it."""
    if t.dim() != 2:
        t = t.reshape(-1, cols) if t.numel() else t.reshape(t.shape[:-1].numel(), cols)
    pitch, step = t.stride()
    if (step != 1 and cols > 1) or (pitch < cols and t.shape[0] > 1):
        t = t.contiguous()
        pitch = cols
    return t, max(pitch, cols)


def _vector(t, n: int, name: str, index: int):
    """An fp32 vector of n values on device `index` (or None)."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.shape != (n,) or t.get_device() != index:
        raise RuntimeError(f"{name}: {n} float32 values on cuda:{index}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t if t.is_contiguous() else t.contiguous()


def _call(index: int, func, *args):
    """func(*args, stream) on the current stream of device `index`."""
    if torch.cuda.current_device() == index:
        status = func(*args, B._raw_stream(index) if B._raw_stream is not None else torch.cuda.current_stream().cuda_stream)
    else:
        with torch.cuda.device(index):
            status = func(*args, torch.cuda.current_stream().cuda_stream)
    if status != B.OK:
        raise B.Int8tError(status)


@functools.lru_cache(maxsize=1024)
def _plan(M: int, K: int, N: int, kind: int, wkind: int):
    """What calls of these sizes have in common: the descriptor, scratch bytes of its directions (forward, backward, served), and where the
    backward pass's codes and scales (of x, of W) lie in one piece of memory, and its size."""
    desc = B.LinearDesc(M, K, N, kind, wkind)
    need = tuple(B.lib.int8t_linear_workspace_bytes(desc, i) for i in range(3))
    at, places = 0, []
    for n in (M * _pad16(K), N * _pad16(K), 4 * M, 4 * N):
        places.append(at)
        at += (n + 255) & ~255
    return desc, need, tuple(places), at


class ServedLinear:
    """A linear layer in use: weights as codes with a scale for each output channel, laid out once; each token gets its scale when it
    arrives.  y = x W^T + b in x's type; no gradients.

    codes: (out, in rounded up to 16) int8, zero beyond in;  scales: (out,) float32"""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, in_features: int, bias: torch.Tensor | None = None):
        if codes.dtype is not torch.int8 or codes.dim() != 2 or codes.shape[1] != _pad16(in_features) or not codes.is_contiguous() or not codes.is_cuda:
            raise RuntimeError(f"codes: contiguous int8 (out, {_pad16(in_features)}) on the device, not {tuple(codes.shape)} of {codes.dtype}")
        self.in_features, self.out_features = int(in_features), codes.shape[0]
        self._index = codes.get_device()
        self._tensors = codes, _vector(scales, codes.shape[0], "scales", self._index), _vector(bias, codes.shape[0], "bias", self._index)
        self._b = B.LinearBuffers(wq=codes.data_ptr(), sw=self.scales.data_ptr(), bias=None if self.bias is None else self.bias.data_ptr(),
                                  y_pitch=self.out_features)

    # (not to be replaced: their addresses are taken once)
    codes = property(lambda self: self._tensors[0])
    scales = property(lambda self: self._tensors[1])
    bias = property(lambda self: self._tensors[2])

    @classmethod
    def of(cls, weight: torch.Tensor, bias: torch.Tensor | None = None) -> "ServedLinear":
        """From floating weights (out, in): nearest codes, c the maximum of a row."""
        if weight.dim() != 2:
            raise RuntimeError(f"weight of {weight.dim()} dimensions")
        kind = _type(weight, "weight")
        N, K = weight.shape
        w, pitch = _rows(weight.detach(), K)
        codes = torch.empty(N, _pad16(K), dtype=torch.int8, device=w.device)
        scales = torch.empty(N, dtype=torch.float32, device=w.device)
        _call(w.get_device(), B.lib.int8t_quantize_rows, w.data_ptr(), kind, N, K, pitch, None, B.ROUND_NEAREST_EVEN, 0, codes.data_ptr(), scales.data_ptr())
        return cls(codes, scales, K, bias)

    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        kind = B.DTYPES.get(x.dtype)
        shape = x.shape
        if kind is None or x.get_device() != self._index or not shape or shape[-1] != self.in_features:
            _type(x, "x")
            raise RuntimeError(f"input of {tuple(shape)} on {x.device} in a layer of {self.in_features} on {self.codes.device}")
        y = torch.empty(shape[:-1] + (self.out_features,), dtype=x.dtype, device=x.device)
        if y.numel() == 0:
            return y
        rows, pitch = _rows(x, self.in_features)
        desc, (_, _, need), _, _ = _plan(rows.shape[0], self.in_features, self.out_features, kind, kind)
        b = B.LinearBuffers.from_buffer_copy(self._b)
        b.x, b.x_pitch, b.y = rows.data_ptr(), pitch, y.data_ptr()
        if need:
            ws = torch.empty(need, dtype=torch.uint8, device=x.device)
            b.ws, b.ws_bytes = ws.data_ptr(), need
        _call(self._index, B.lib.int8t_linear_fwd, desc, b)
        return y


class _LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, seed):
        kind, wkind = _type(x, "x"), _type(w, "weight")
        shape = x.shape
        if w.dim() != 2 or not shape or shape[-1] != w.shape[1] or w.device != x.device:
            raise RuntimeError(f"input of {tuple(shape)} on {x.device}, weight of {tuple(w.shape)} on {w.device}")
        N, K = w.shape
        index, dev = x.get_device(), x.device
        bias = _vector(bias, N, "bias", index)
        (rows, pitch), (wr, w_pitch) = _rows(x, K), _rows(w, K)
        M = rows.shape[0]
        y = torch.empty(shape[:-1] + (N,), dtype=x.dtype, device=dev)
        # codes and scales of x and W, in one piece of memory: the backward pass reads them
        desc, (need, later, _), places, size = _plan(M, K, N, kind, wkind)
        kept = torch.empty(size, dtype=torch.uint8, device=dev)
        at = kept.data_ptr()
        b = B.LinearBuffers()
        b.xq, b.wq, b.sx, b.sw = at, at + places[1], at + places[2], at + places[3]
        if M:
            b.x, b.x_pitch, b.w, b.w_pitch, b.y, b.y_pitch = rows.data_ptr(), pitch, wr.data_ptr(), w_pitch, y.data_ptr(), N
            if bias is not None:
                b.bias = bias.data_ptr()
            if need:
                ws = torch.empty(need, dtype=torch.uint8, device=dev)
                b.ws, b.ws_bytes = ws.data_ptr(), need
            _call(index, B.lib.int8t_linear_fwd, desc, b)
        ctx.save_for_backward(kept)
        ctx.desc, ctx.need, ctx.places, ctx.seed, ctx.x_shape, ctx.w_dtype = desc, later, places, seed, shape, w.dtype
        return y

    @staticmethod
    def backward(ctx, dy):
        if torch.is_grad_enabled():
            raise RuntimeError("linear() is differentiable once")
        if _transformed() and _tangent(dy):
            raise RuntimeError("linear() has no forward mode, its gradient neither")
        want_x, want_w, want_b = ctx.needs_input_grad[:3]
        desc, dev = ctx.desc, dy.device
        M, K, N = desc.M, desc.K, desc.N
        dx = torch.empty(ctx.x_shape, dtype=dy.dtype, device=dev) if want_x else None
        if M == 0:
            return (dx, torch.zeros(N, K, dtype=ctx.w_dtype, device=dev) if want_w else None,
                    torch.zeros(N, dtype=torch.float32, device=dev) if want_b else None, None)
        g, pitch = _rows(dy, N)
        kept, = ctx.saved_tensors
        b = B.LinearBuffers()
        at, places = kept.data_ptr(), ctx.places
        b.xq, b.wq, b.sx, b.sw = at, at + places[1], at + places[2], at + places[3]
        b.dy, b.dy_pitch = g.data_ptr(), pitch
        if want_x:
            b.dx = dx.data_ptr()
        dw = db = None
        if want_w:
            dw = torch.empty(N, K, dtype=ctx.w_dtype, device=dev)
            b.dw = dw.data_ptr()
        if want_b:
            db = torch.empty(N, dtype=torch.float32, device=dev)
            b.db = db.data_ptr()
        need = ctx.need
        ws = torch.empty(need, dtype=torch.uint8, device=dev)
        b.ws, b.ws_bytes = ws.data_ptr(), need
        _call(dy.get_device(), B.lib.int8t_linear_bwd, desc, b, ctx.seed)
        return dx, dw, db, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, seed: int = 0) -> torch.Tensor:
    """x W^T + b with a scale for each token and output channel, differentiable (once): the gradients' codes are rounded stochastically with
    draws of `seed` (Eq.3), the scales of the summed axis in them.  x (.., in) and weight (out, in) fp32, bf16 or fp16; bias fp32."""
    return _LinearFn.apply(x, weight, bias, int(seed) & 0xFFFFFFFFFFFFFFFF)


class TokenLinear(torch.nn.Module):
    """Drop-in for `torch.nn.Linear` through linear(): scales per token and output channel instead of per tensor (`Int8Linear`).  The
    bias stays fp32.  As there, the stream of seeds starts at a hash of the layer's name and advances by one per forward pass that
    keeps codes for a backward pass."""

    def __init__(self, in_features, out_features, bias=True, dtype=torch.float32, device="cuda:0", seed: int | None = None, name: str = ""):
        super().__init__()
        self.in_features, self.out_features = in_features, out_features
        w = torch.randn(out_features, in_features, device=device) * (1.0 / in_features) ** 0.5
        self.weight = torch.nn.Parameter(w.to(dtype))
        self.bias = torch.nn.Parameter(torch.zeros(out_features, device=device)) if bias else None
        self._seed = int(seed) if seed is not None else (zlib.crc32(name.encode()) << 20 if name else 0)

    def forward(self, x):
        if torch.is_grad_enabled():
            self._seed += 1
        return linear(x, self.weight, self.bias, self._seed)

    def served(self) -> ServedLinear:
        """The layer with its present weights, for use without gradients."""
        return ServedLinear.of(self.weight, self.bias if self.bias is None else self.bias.detach())


class PagedCache:
    """Keys and values in 8 bits with a scale for each token and head, in pages: place `slot` is row slot % page_size of page
    slot // page_size.

    kq, vq: (pages, heads, page_size, dim) int8;  ks, vs: (pages, heads, page_size) float32"""

    _calls = B.lib.int8t_cache_write, B.lib.int8t_cache_read, B.lib.int8t_cache_attend_workspace_bytes, B.lib.int8t_cache_attend

    def __init__(self, kq, ks, vq, vs):
        if kq.dim() != 4 or kq.shape != vq.shape or ks.shape != kq.shape[:3] or vs.shape != ks.shape:
            raise RuntimeError(f"cache of codes {tuple(kq.shape)}, {tuple(vq.shape)} and scales {tuple(ks.shape)}, {tuple(vs.shape)}")
        for t, kind, name in ((kq, torch.int8, "kq"), (vq, torch.int8, "vq"), (ks, torch.float32, "ks"), (vs, torch.float32, "vs")):
            if t.dtype is not kind or not t.is_cuda or not t.is_contiguous() or t.device != kq.device:
                raise RuntimeError(f"{name}: contiguous {kind} on {kq.device}")
        self._keep(B.Cache, kq, ks, vq, vs, kq.shape[3])

    def _keep(self, struct, kq, ks, vq, vs, dim):
        self._tensors = kq, ks, vq, vs
        (self.pages, self.heads, self.page_size), self.dim = kq.shape[:3], dim
        if self.dim % 16 or not 0 < self.dim <= 256:
            raise RuntimeError(f"head dimension {self.dim}: a multiple of 16, at most 256")
        self._index, self._plans = kq.get_device(), {}
        self._c = struct(kq.data_ptr(), vq.data_ptr(), ks.data_ptr(), vs.data_ptr(), self.pages, self.page_size, self.heads, self.dim)

    # (not to be replaced: their addresses are taken once)
    kq = property(lambda self: self._tensors[0])
    ks = property(lambda self: self._tensors[1])
    vq = property(lambda self: self._tensors[2])
    vs = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, pages: int, page_size: int, heads: int, dim: int, device="cuda:0") -> "PagedCache":
        q = [torch.zeros(pages, heads, page_size, dim, dtype=torch.int8, device=device) for _ in range(2)]
        s = [torch.zeros(pages, heads, page_size, dtype=torch.float32, device=device) for _ in range(2)]
        return cls(q[0], s[0], q[1], s[1])

    def _slots(self, slots):
        if slots.dtype is not torch.int64 or slots.dim() != 1 or slots.get_device() != self._index:
            raise RuntimeError(f"slots: int64 vector on {self.kq.device}")
        return slots if slots.is_contiguous() else slots.contiguous()

    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """Token t's rows k[t], v[t] (tokens, heads, dim) to place slots[t], quantised; a slot below 0 leaves its token out."""
        kind = B.DTYPES.get(k.dtype)
        shape = k.shape
        if (kind is None or v.dtype is not k.dtype or shape != v.shape or len(shape) != 3 or shape[1] != self.heads or shape[2] != self.dim
                or k.get_device() != self._index or v.get_device() != self._index):
            _type(k, "k")
            raise RuntimeError(f"k {tuple(shape)} of {k.dtype}, v {tuple(v.shape)} of {v.dtype} in a cache of {self.heads} heads of {self.dim} on {self.kq.device}")
        slots = self._slots(slots)
        if slots.shape[0] != shape[0]:
            raise RuntimeError(f"{slots.shape[0]} slots for {shape[0]} tokens")
        (kt, kh, kd), (vt, vh, vd) = k.stride(), v.stride()
        if kd != 1:
            k = k.contiguous()
            kt, kh, _ = k.stride()
        if vd != 1:
            v = v.contiguous()
            vt, vh, _ = v.stride()
        _call(self._index, self._calls[0], self._c, k.data_ptr(), v.data_ptr(), kind, shape[0], kt, kh, vt, vh, slots.data_ptr())

    def read(self, slots: torch.Tensor, dtype=torch.float32):
        """(k, v), each (len(slots), heads, dim), as the cache holds them; zeros for slots outside it."""
        kind = B.DTYPES.get(dtype)
        if kind is None:
            raise TypeError(f"{dtype}: float32, bfloat16 or float16")
        slots = self._slots(slots)
        n = slots.shape[0]
        k = torch.empty((n, self.heads, self.dim), dtype=dtype, device=slots.device)
        v = torch.empty_like(k)
        _call(self._index, self._calls[1], self._c, slots.data_ptr(), n, k.data_ptr(), v.data_ptr(), kind)
        return k, v

    def attend(self, q: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, causal: bool = True,
               scale: float | None = None, longest: int | None = None, return_lse: bool = False):
        """Attention of new tokens, (tokens, query heads, dim), over the pages of their requests: request b's are
        starts[b] .. starts[b + 1] - 1 and see the first lengths[b] keys of pages table[b], causal: each up to its own place (the last
        new token sees all).  Query heads are a multiple of the cache's; head h goes with h // group.  `longest`: no length is larger
        (a guide for the division of the work, by which sums are ordered).  int32 starts (requests + 1), lengths (requests), table (requests, width).
        A token that sees nothing gets zeros (logarithm of its sum: -inf); what tokens before the first request's or behind the last one's get is not
        defined.  No gradients."""
        kind = B.DTYPES.get(q.dtype)
        shape, index = q.shape, self._index
        if kind is None or len(shape) != 3 or shape[2] != self.dim or shape[1] % self.heads or shape[1] == 0 or q.get_device() != index:
            _type(q, "q")
            raise RuntimeError(f"q {tuple(shape)} on {q.device} over a cache of {self.heads} heads of {self.dim} on {self.kq.device}")
        T, heads, dim = shape
        n, wide = lengths.numel(), table.shape
        if lengths.dim() != 1 or starts.shape != (n + 1,) or len(wide) != 2 or wide[0] != n:
            raise RuntimeError(f"starts {tuple(starts.shape)}, lengths {tuple(lengths.shape)}, table {tuple(wide)}")
        i32 = torch.int32
        if not (starts.dtype is i32 and lengths.dtype is i32 and table.dtype is i32 and starts.get_device() == lengths.get_device() == table.get_device() == index):
            for t in (starts, lengths, table):
                if t.dtype is not i32 or t.get_device() != index:
                    raise RuntimeError(f"starts, lengths, table: int32 on {q.device}, not {t.dtype} on {t.device}")
        token, head, step = q.stride()
        if step != 1:
            q = q.contiguous()
            token, head, _ = q.stride()
        pitch, step = table.stride()
        if (step != 1 and wide[1] > 1) or (pitch < wide[1] and n > 1):
            table = table.contiguous()
            pitch = wide[1]
        if not (starts.is_contiguous() and lengths.is_contiguous()):
            starts, lengths = starts.contiguous(), lengths.contiguous()
        out = torch.empty_like(q) if q.is_contiguous() else q.new_empty(shape)
        lse = torch.empty((T, heads), dtype=torch.float32, device=q.device) if return_lse else None
        if T:
            # (descriptors and scratch bytes of the last calls' sizes)
            key = T, n, heads, wide[1], 0 if longest is None else max(1, int(longest)), kind, 1 if causal else 0, dim ** -0.5 if scale is None else float(scale), token, head, pitch
            plan = self._plans.get(key)
            if plan is None:
                d = B.AttendDesc(T, n, heads // self.heads, *key[3:10], max(pitch, wide[1]))
                if len(self._plans) >= 256:
                    self._plans.clear()
                plan = self._plans[key] = d, self._calls[2](self._c, d)
            d, need = plan
            ws = torch.empty(need, dtype=torch.uint8, device=q.device) if need else None
            _call(index, self._calls[3], self._c, d, q.data_ptr(), starts.data_ptr(), lengths.data_ptr(), table.data_ptr(), out.data_ptr(),
                  None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(), need)
        return (out, lse) if return_lse else out
