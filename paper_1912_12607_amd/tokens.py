"""Token operators over the C ABI: linear layers with a scale for each token and output channel (for training and for serving), a
paged cache of keys and values in 8 bits, and attention of new tokens over it.

Plumbing only, as in ``autograd``: every arithmetic step is one of the library's entry points; torch supplies device memory, the current
stream and the autograd graph.  CUDA(ROCm) tensors in fp32, bf16 or fp16.

    layer = ServedLinear.of(weight, bias)               # codes and scales, laid out once
    cache = PagedCache.empty(pages, page_size, heads, dim, device)
    cache.write(k, v, slots)                            # quantised on the way in
    o = cache.attend(q, starts, lengths, table)         # the new tokens of each request over its pages
    y = linear(x, weight, bias, seed=7)                 # differentiable; TokenLinear is the module
"""
from __future__ import annotations

import math
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


def _rows(t: torch.Tensor, cols: int) -> torch.Tensor:
    """t as rows of `cols` contiguous values; a copy where its strides do not allow it."""
    if t.dim() != 2:
        t = t.reshape(-1, cols) if cols else t.reshape(t.shape[:-1].numel(), 0)
    if t.shape[0] > 1 and t.stride(0) < cols or t.shape[1] > 1 and t.stride(1) != 1:
        t = t.contiguous()
    return t


def _pitch(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else max(t.shape[1], t.stride(0))


def _vector(t, n: int, name: str, like: torch.Tensor):
    """An fp32 vector of n values on like's device (or None)."""
    if t is None:
        return None
    if t.dtype is not torch.float32 or t.dim() != 1 or t.shape[0] != n or t.device != like.device:
        raise RuntimeError(f"{name}: {n} float32 values on {like.device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
    return t.contiguous()


def _scratch(nbytes: int, dev) -> torch.Tensor:
    return torch.empty(max(nbytes, 16), dtype=torch.uint8, device=dev)


class ServedLinear:
    """A linear layer in use: weights as codes with a scale for each output channel, laid out once; each token gets its scale when it
    arrives.  y = x W^T + b in x's type; no gradients.

    codes: (out, in rounded up to 16) int8, zero beyond in;  scales: (out,) float32"""

    def __init__(self, codes: torch.Tensor, scales: torch.Tensor, in_features: int, bias: torch.Tensor | None = None):
        if codes.dtype is not torch.int8 or codes.dim() != 2 or codes.shape[1] != _pad16(in_features) or not codes.is_contiguous() or not codes.is_cuda:
            raise RuntimeError(f"codes: contiguous int8 (out, {_pad16(in_features)}) on the device, not {tuple(codes.shape)} of {codes.dtype}")
        self.in_features, self.out_features = int(in_features), codes.shape[0]
        self.codes, self.scales = codes, _vector(scales, codes.shape[0], "scales", codes)
        self.bias = _vector(bias, codes.shape[0], "bias", codes)

    @classmethod
    def of(cls, weight: torch.Tensor, bias: torch.Tensor | None = None) -> "ServedLinear":
        """From floating weights (out, in): nearest codes, c the maximum of a row."""
        if weight.dim() != 2:
            raise RuntimeError(f"weight of {weight.dim()} dimensions")
        w = _rows(weight.detach(), weight.shape[1])
        N, K = w.shape
        codes = torch.empty(N, _pad16(K), dtype=torch.int8, device=w.device)
        scales = torch.empty(N, dtype=torch.float32, device=w.device)
        kind = _type(w, "weight")
        with torch.cuda.device(w.device):
            B._check(B.lib.int8t_quantize_rows(w.data_ptr(), kind, N, K, _pitch(w), None, B.ROUND_NEAREST_EVEN, 0, codes.data_ptr(), scales.data_ptr(), B._stream(None)))
        return cls(codes, scales, K, bias)

    @torch.no_grad()
    def __call__(self, x: torch.Tensor) -> torch.Tensor:
        kind = _type(x, "x")
        if x.dim() < 1 or x.shape[-1] != self.in_features or x.device != self.codes.device:
            raise RuntimeError(f"input of {tuple(x.shape)} on {x.device} in a layer of {self.in_features} on {self.codes.device}")
        y = torch.empty(x.shape[:-1] + (self.out_features,), dtype=x.dtype, device=x.device)
        if y.numel() == 0:
            return y
        rows = _rows(x, self.in_features)
        desc = B.LinearDesc(rows.shape[0], self.in_features, self.out_features, kind, kind)
        ws = _scratch(B.int8t_linear_workspace_bytes(desc, 0), x.device)
        b = B.LinearBuffers(x=rows.data_ptr(), x_pitch=_pitch(rows), wq=self.codes.data_ptr(), sw=self.scales.data_ptr(),
                            bias=None if self.bias is None else self.bias.data_ptr(), y=y.data_ptr(), y_pitch=self.out_features,
                            ws=ws.data_ptr(), ws_bytes=ws.numel())
        with torch.cuda.device(x.device):
            B.int8t_linear_fwd(desc, b)
        return y


class _LinearFn(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, seed):
        kind, wkind = _type(x, "x"), _type(w, "weight")
        if w.dim() != 2 or x.dim() < 1 or x.shape[-1] != w.shape[1] or w.device != x.device:
            raise RuntimeError(f"input of {tuple(x.shape)} on {x.device}, weight of {tuple(w.shape)} on {w.device}")
        N, K = w.shape
        bias = _vector(bias, N, "bias", x)
        rows, wr = _rows(x, K), _rows(w, K)
        M, dev = rows.shape[0], x.device
        y = torch.empty(x.shape[:-1] + (N,), dtype=x.dtype, device=dev)
        desc = B.LinearDesc(M, K, N, kind, wkind)
        xq = torch.empty(M, _pad16(K), dtype=torch.int8, device=dev)
        wq = torch.empty(N, _pad16(K), dtype=torch.int8, device=dev)
        sx = torch.empty(M, dtype=torch.float32, device=dev)
        sw = torch.empty(N, dtype=torch.float32, device=dev)
        if M:
            ws = _scratch(B.int8t_linear_workspace_bytes(desc, 0), dev)
            b = B.LinearBuffers(x=rows.data_ptr(), x_pitch=_pitch(rows), w=wr.data_ptr(), w_pitch=_pitch(wr), xq=xq.data_ptr(), wq=wq.data_ptr(),
                                sx=sx.data_ptr(), sw=sw.data_ptr(), bias=None if bias is None else bias.data_ptr(), y=y.data_ptr(), y_pitch=N,
                                ws=ws.data_ptr(), ws_bytes=ws.numel())
            with torch.cuda.device(dev):
                B.int8t_linear_fwd(desc, b)
        ctx.save_for_backward(xq, sx, wq, sw)
        ctx.desc, ctx.seed, ctx.x_shape, ctx.w_dtype = desc, seed, x.shape, w.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        want_x, want_w, want_b = ctx.needs_input_grad[:3]
        desc = ctx.desc
        g = _rows(dy, desc.N)
        dx = torch.empty(ctx.x_shape, dtype=dy.dtype, device=dy.device) if want_x else None
        dw = db = None
        if desc.M == 0:
            dw = torch.zeros(desc.N, desc.K, dtype=ctx.w_dtype, device=dy.device) if want_w else None
            db = torch.zeros(desc.N, dtype=torch.float32, device=dy.device) if want_b else None
            return dx, dw, db, None
        if want_w:
            dw = torch.empty(desc.N, desc.K, dtype=ctx.w_dtype, device=dy.device)
        if want_b:
            if not want_w:                      # (with the weights' gradient the sums come out of its pass over dy)
                db = g.sum(0, dtype=torch.float32)
            else:
                db = torch.empty(desc.N, dtype=torch.float32, device=dy.device)
        if not (want_x or want_w):
            return None, None, db, None
        xq, sx, wq, sw = ctx.saved_tensors
        ws = _scratch(B.int8t_linear_workspace_bytes(desc, 1), dy.device)
        b = B.LinearBuffers(dy=g.data_ptr(), dy_pitch=_pitch(g), xq=xq.data_ptr(), wq=wq.data_ptr(), sx=sx.data_ptr(), sw=sw.data_ptr(),
                            dx=dx.data_ptr() if want_x else None, dw=dw.data_ptr() if want_w else None,
                            db=db.data_ptr() if want_b and want_w else None, ws=ws.data_ptr(), ws_bytes=ws.numel())
        with torch.cuda.device(dy.device):
            B.int8t_linear_bwd(desc, b, ctx.seed)
        return dx, dw, db, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: torch.Tensor | None = None, seed: int = 0) -> torch.Tensor:
    """x W^T + b with a scale for each token and output channel, differentiable: the gradients' codes are rounded stochastically with
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

    def __init__(self, kq, ks, vq, vs):
        if kq.dim() != 4 or kq.shape != vq.shape or ks.shape != kq.shape[:3] or vs.shape != ks.shape:
            raise RuntimeError(f"cache of codes {tuple(kq.shape)}, {tuple(vq.shape)} and scales {tuple(ks.shape)}, {tuple(vs.shape)}")
        for t, kind, name in ((kq, torch.int8, "kq"), (vq, torch.int8, "vq"), (ks, torch.float32, "ks"), (vs, torch.float32, "vs")):
            if t.dtype is not kind or not t.is_cuda or not t.is_contiguous() or t.device != kq.device:
                raise RuntimeError(f"{name}: contiguous {kind} on {kq.device}")
        self.kq, self.ks, self.vq, self.vs = kq, ks, vq, vs
        self.pages, self.heads, self.page_size, self.dim = kq.shape
        if self.dim % 16 or not 0 < self.dim <= 256:
            raise RuntimeError(f"head dimension {self.dim}: a multiple of 16, at most 256")
        self._c = B.Cache(kq.data_ptr(), vq.data_ptr(), ks.data_ptr(), vs.data_ptr(), self.pages, self.page_size, self.heads, self.dim)

    @classmethod
    def empty(cls, pages: int, page_size: int, heads: int, dim: int, device="cuda:0") -> "PagedCache":
        q = [torch.zeros(pages, heads, page_size, dim, dtype=torch.int8, device=device) for _ in range(2)]
        s = [torch.zeros(pages, heads, page_size, dtype=torch.float32, device=device) for _ in range(2)]
        return cls(q[0], s[0], q[1], s[1])

    def _slots(self, slots):
        if slots.dtype is not torch.int64 or slots.dim() != 1 or slots.device != self.kq.device:
            raise RuntimeError(f"slots: int64 vector on {self.kq.device}")
        return slots.contiguous()

    @torch.no_grad()
    def write(self, k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor) -> None:
        """Token t's rows k[t], v[t] (tokens, heads, dim) to place slots[t], quantised; a slot below 0 leaves its token out."""
        kind = _type(k, "k")
        if k.shape != v.shape or k.dtype != v.dtype or k.dim() != 3 or k.shape[1:] != (self.heads, self.dim) or k.device != self.kq.device or v.device != k.device:
            raise RuntimeError(f"k {tuple(k.shape)}, v {tuple(v.shape)} in a cache of {self.heads} heads of {self.dim}")
        slots = self._slots(slots)
        if slots.shape[0] != k.shape[0]:
            raise RuntimeError(f"{slots.shape[0]} slots for {k.shape[0]} tokens")
        k, v = (t if t.stride(2) == 1 and min(t.stride()[:2]) >= 0 else t.contiguous() for t in (k, v))
        with torch.cuda.device(k.device):
            B._check(B.lib.int8t_cache_write(self._c, k.data_ptr(), v.data_ptr(), kind, k.shape[0], k.stride(0), k.stride(1), v.stride(0), v.stride(1),
                                             slots.data_ptr(), B._stream(None)))

    @torch.no_grad()
    def read(self, slots: torch.Tensor, dtype=torch.float32):
        """(k, v), each (len(slots), heads, dim), as the cache holds them; zeros for slots outside it."""
        if dtype not in B.DTYPES:
            raise TypeError(f"{dtype}: float32, bfloat16 or float16")
        slots = self._slots(slots)
        k, v = (torch.empty(slots.shape[0], self.heads, self.dim, dtype=dtype, device=self.kq.device) for _ in range(2))
        with torch.cuda.device(self.kq.device):
            B._check(B.lib.int8t_cache_read(self._c, slots.data_ptr(), slots.shape[0], k.data_ptr(), v.data_ptr(), B.DTYPES[dtype], B._stream(None)))
        return k, v

    @torch.no_grad()
    def attend(self, q: torch.Tensor, starts: torch.Tensor, lengths: torch.Tensor, table: torch.Tensor, causal: bool = True,
               scale: float | None = None, longest: int | None = None, return_lse: bool = False):
        """Attention of new tokens, (tokens, query heads, dim), over the pages of their requests: request b's are
        starts[b] .. starts[b + 1] - 1 and see the first lengths[b] keys of pages table[b], causal: each up to its own place (the last
        new token sees all).  Query heads are a multiple of the cache's; head h goes with h // group.  `longest`: no length is larger
        (divides the work; the result does not depend on it).  int32 starts (requests + 1), lengths (requests), table (requests, width).
        A token that sees nothing gets zeros (logarithm of its sum: -inf)."""
        kind = _type(q, "q")
        if q.dim() != 3 or q.shape[2] != self.dim or q.shape[1] % self.heads or q.shape[1] == 0 or q.device != self.kq.device:
            raise RuntimeError(f"q {tuple(q.shape)} on {q.device} over a cache of {self.heads} heads of {self.dim} on {self.kq.device}")
        n = lengths.shape[0] if lengths.dim() == 1 else -1
        if starts.shape != (n + 1,) or table.dim() != 2 or table.shape[0] != n:
            raise RuntimeError(f"starts {tuple(starts.shape)}, lengths {tuple(lengths.shape)}, table {tuple(table.shape)}")
        for t, name in ((starts, "starts"), (lengths, "lengths"), (table, "table")):
            if t.dtype is not torch.int32 or t.device != q.device:
                raise RuntimeError(f"{name}: int32 on {q.device}")
        if q.stride(2) != 1 or min(q.stride()[:2]) < 0:
            q = q.contiguous()
        if table.shape[1] > 1 and table.stride(1) != 1 or table.shape[0] > 1 and table.stride(0) < table.shape[1]:
            table = table.contiguous()
        starts, lengths = starts.contiguous(), lengths.contiguous()
        T, heads = q.shape[:2]
        out = torch.empty(T, heads, self.dim, dtype=q.dtype, device=q.device)
        lse = torch.empty(T, heads, dtype=torch.float32, device=q.device) if return_lse else None
        if T:
            d = B.AttendDesc(T, n, heads // self.heads, table.shape[1], 0 if longest is None else max(1, int(longest)), kind, int(bool(causal)),
                             1.0 / math.sqrt(self.dim) if scale is None else float(scale), q.stride(0), q.stride(1), _pitch(table))
            need = B.lib.int8t_cache_attend_workspace_bytes(self._c, d)
            ws = _scratch(need, q.device) if need else None
            with torch.cuda.device(q.device):
                B._check(B.lib.int8t_cache_attend(self._c, d, q.data_ptr(), starts.data_ptr(), lengths.data_ptr(), table.data_ptr(), out.data_ptr(),
                                                  None if lse is None else lse.data_ptr(), None if ws is None else ws.data_ptr(), need, B._stream(None)))
        return (out, lse) if return_lse else out
