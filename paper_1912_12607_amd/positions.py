"""What stands between a layer and a paged cache, over the C ABI: rotary positions of queries and keys (for training and for serving), and the pages, slots and
positions of a batch's new tokens, found on the GPU.

Plumbing only, as in ``tokens``: the arithmetic is the library's.

    rotary = Rotary(128, layout="half", factor=8.0, original=8192)
    q, k = rotary(q, k, positions)                      # differentiable; rotary.turn_(q, k, positions) in place
    pages = PageTable.empty(requests, width, pages, page_size)
    step = pages.extend(new, tokens)                    # step.slots, .positions, .starts, .lengths: what cache.write, rotary and cache.attend take
    pages.accept(step)                                  # the new tokens stay; pages.shrink(lengths) takes tokens and their pages back
"""
from __future__ import annotations

import math
from typing import NamedTuple

import torch

from . import binding as B
from .tokens import _call, _tangent, _transformed, _type


class _RotateFn(torch.autograd.Function):
    """back: by the negative angles.  A turn is linear: gradients are turned back, tangents as what they belong to."""

    @staticmethod
    def forward(ctx, rotary, positions, q, k, back):
        ctx.rotary, ctx.two, ctx.plan, ctx.back = rotary, k is not None, rotary._check(q, k, positions), back
        ctx.shapes = (q.shape, k.shape) if ctx.two else (q.shape,)
        ctx.save_for_backward(positions)
        ctx.save_for_forward(positions)
        ctx.set_materialize_grads(False)
        out = rotary._turn(ctx.plan, q, k, positions, back)
        return out if ctx.two else out[0]

    @staticmethod
    def jvp(ctx, _rotary, _positions, q, k, _back):
        positions, = ctx.saved_tensors
        tangents = (q, k) if ctx.two else (q,)
        there = [t for t in tangents if t is not None]
        turned = _RotateFn.apply(ctx.rotary, positions, there[0], there[1] if len(there) > 1 else None, ctx.back)
        turned = iter(turned if len(there) > 1 else (turned,))
        out = [next(turned) if t is not None else there[0].new_zeros(shape) for t, shape in zip(tangents, ctx.shapes)]
        return tuple(out) if ctx.two else out[0]

    @staticmethod
    def backward(ctx, *grads):
        if torch.is_grad_enabled():
            raise RuntimeError("a Rotary is differentiable once")
        positions, = ctx.saved_tensors
        want = [g if n else None for g, n in zip(grads, ctx.needs_input_grad[2:4])]
        there = [g for g in want if g is not None]
        if not there:
            return None, None, None, None, None
        second = there[1] if len(there) > 1 else None
        if _transformed():                       # (gradients may have tangents)
            turned = _RotateFn.apply(ctx.rotary, positions, there[0], second, 1 - ctx.back)
            turned = iter(turned if second is not None else (turned,))
        else:
            plan = ctx.plan if len(there) == 1 + ctx.two else ctx.rotary._check(there[0], None, positions)
            turned = iter(ctx.rotary._turn(plan, there[0], second, positions, 1 - ctx.back))
        out = [next(turned) if g is not None else None for g in want]
        return (None, None, out[0], out[1] if ctx.two else None, None)


class Rotary:
    """Rotary positions: pair i of a head's first `rot` values turns by the angle position * frequency[i], frequency[i] = base^(-2 i / rot).

    layout: "half" (pairs i and i + rot / 2) or "interleaved" (2 i and 2 i + 1).  For contexts longer than trained ones: `factor` divides the frequencies; with
    `original` (the length trained for) only those of pairs that turn less than `slow` times over it, while pairs that turn more than `fast` times keep theirs and the
    ones between go over from one to the other in proportion to their turns.  `amplitude` multiplies the result's turned values.  Frequencies and angles are formed in
    64 bits.  `frequencies`: rot / 2 of the caller's own, in radians per position, instead of all that."""

    def __init__(self, rot: int, base: float = 10000.0, layout: str = "half", factor: float = 1.0, original: int = 0, slow: float = 1.0, fast: float = 32.0,
                 amplitude: float = 1.0, frequencies=None):
        if rot <= 0 or rot % 2:
            raise ValueError(f"rot = {rot}: an even number of values")
        if layout not in ("half", "interleaved"):
            raise ValueError(f"layout {layout!r}: half or interleaved")
        if frequencies is None:
            if not (base > 0.0 and factor > 0.0 and original >= 0 and 0.0 <= slow < fast):
                raise ValueError(f"base {base}, factor {factor}, original {original}, slow {slow}, fast {fast}")
            f = float(base) ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
            if original:
                keep = ((f * (original / (2.0 * math.pi)) - slow) / (fast - slow)).clamp(0.0, 1.0)
                f = f * (keep + (1.0 - keep) / factor)
            else:
                f = f / factor
        else:
            f = torch.as_tensor(frequencies, dtype=torch.float64, device="cpu")
            if f.shape != (rot // 2,):
                raise ValueError(f"frequencies of shape {tuple(f.shape)}: {rot // 2}")
        if not math.isfinite(amplitude):
            raise ValueError(f"amplitude {amplitude}")
        self._parameters = int(rot), layout, float(amplitude), f.clone()
        self._turns = {}                     # device -> turns per position
        self._plans = {}                     # shapes and type -> descriptors

    # (not to be replaced: calls keep what they made of them)
    rot = property(lambda self: self._parameters[0])
    layout = property(lambda self: self._parameters[1])
    amplitude = property(lambda self: self._parameters[2])
    frequencies = property(lambda self: self._parameters[3].clone())

    def _on(self, device):
        t = self._turns.get(device)
        if t is None:
            t = self._turns[device] = (self._parameters[3] / (2.0 * math.pi)).to(device)
        return t

    def to(self, device) -> "Rotary":
        """Lays the frequencies out on the device (a captured graph's first call would copy them)."""
        device = torch.device(device)
        self._on(torch.device("cuda", torch.cuda.current_device()) if device.type == "cuda" and device.index is None else device)
        return self

    def _check(self, q, k, positions):
        """What calls of these shapes have in common: (descriptors, tokens, heads of q and k, dim), looked up after the first."""
        shape, device = q.shape, q.device
        if positions.dtype is not torch.int32 or positions.shape != shape[:-2] or positions.device != device:
            _type(q, "q")
            raise RuntimeError(f"positions {tuple(positions.shape)} of {positions.dtype} on {positions.device}: int32 {tuple(shape[:-2])} on {device}")
        kind = q.dtype
        if k is None:
            key = shape, kind
        else:
            key = shape, kind, k.shape
            if k.dtype is not kind or k.device != device:
                raise RuntimeError(f"k of {k.dtype} on {k.device}, q of {kind} on {device}")
        plan = self._plans.get(key)
        if plan is None:
            code = _type(q, "q")
            for t, name in ((q, "q"), (k, "k")):
                if t is not None and (t.dim() < 3 or t.shape[:-2] != shape[:-2] or t.shape[-1] != shape[-1] or t.shape[-2] == 0):
                    raise RuntimeError(f"{name} {tuple(t.shape)}: (.., heads, dim) as q, {tuple(shape)}")
            if self.rot > shape[-1]:
                raise RuntimeError(f"heads of {shape[-1]} values, {self.rot} of them turned")
            tokens = positions.numel()
            descs = tuple(B.RotateDesc(tokens, shape[-1], self.rot, code, 1 if self.layout == "interleaved" else 0, back, self.amplitude) for back in (0, 1))
            if len(self._plans) >= 1024:
                self._plans.clear()
            plan = self._plans[key] = descs, tokens, (shape[-2], 0 if k is None else k.shape[-2]), shape[-1]
        elif not q.is_cuda:
            _type(q, "q")
        return plan

    @staticmethod
    def _tensor(x, y, heads, dim):
        row = heads * dim
        if x.is_contiguous():
            return B.RotateTensor(x.data_ptr(), y.data_ptr(), row, dim, row, dim, heads)
        token, head, _ = x.stride()
        return B.RotateTensor(x.data_ptr(), y.data_ptr(), token, head, *((token, head) if y is x else (row, dim)), heads)

    def _launch(self, plan, first, second, positions, back):
        """first, second: (source, result) each, or None."""
        if plan[1] == 0:
            return
        if not positions.is_contiguous():
            positions = positions.contiguous()
        x = first[0]
        heads, dim = plan[2:]
        _call(x.get_device(), B.lib.int8t_rotate, plan[0][back], self._tensor(*first, heads[0], dim), None if second is None else self._tensor(*second, heads[1], dim),
              positions.data_ptr(), self._on(x.device).data_ptr())

    @staticmethod
    def _result(x):
        """(source, result): contiguous, the source a tensor that _tensor() takes."""
        if x.is_contiguous():
            return x, torch.empty_like(x)
        if x.stride(-1) != 1 or x.dim() != 3:
            x = x.contiguous()
        return x, x.new_empty(x.shape)

    def _turn(self, plan, q, k, positions, back):
        q, yq = self._result(q)
        yk = None
        if k is not None:
            k, yk = self._result(k)
        self._launch(plan, (q, yq), None if k is None else (k, yk), positions, back)
        return (yq,) if k is None else (yq, yk)

    def __call__(self, q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor):
        """(q, k) turned, or q alone where k is None: (.., heads, dim) of one type, int32 positions (..).  Differentiable (once, and in forward mode); a pass that is captured
        into a CUDA graph takes leaves of which no eager autograd graph lives any more, as linear4()."""
        if (torch.is_grad_enabled() and (q.requires_grad or (k is not None and k.requires_grad))) or _transformed():
            return _RotateFn.apply(self, positions, q, k, 0)
        out = self._turn(self._check(q, k, positions), q, k, positions, 0)
        return out if k is not None else out[0]

    def turn_(self, q: torch.Tensor, k: torch.Tensor | None, positions: torch.Tensor) -> None:
        """The same in place, without gradients: q and k (tokens, heads, dim) in any strides whose heads are contiguous, or contiguous (.., heads, dim)."""
        plan = self._check(q, k, positions)
        for x in (q, k):
            if x is None:
                continue
            if (x.requires_grad and torch.is_grad_enabled()) or (_transformed() and _tangent(x)):
                raise RuntimeError("turn_ has no gradients")
            if not x.is_contiguous() and (x.stride(-1) != 1 or x.dim() != 3 or _overlaps(x)):
                raise RuntimeError(f"in place with strides {x.stride()} of {tuple(x.shape)}")
        if k is not None and _share(q, k):
            raise RuntimeError("q and k share memory")
        self._launch(plan, (q, q), None if k is None else (k, k), positions, 0)
        for x in (q, k):                         # (a graph that has kept one of them for its backward pass will notice)
            if x is not None:
                torch.autograd.graph.increment_version(x)


def _overlaps(x):
    """Whether elements of x share memory (strides sorted: each at least the extent below it)."""
    extent = 1
    for n, s in sorted(zip(x.shape, x.stride()), key=lambda t: t[1]):
        if n > 1 and s < extent:
            return True
        extent = max(extent, s * (n - 1) + extent) if n > 1 else extent
    return False


def _share(q, k):
    """Whether heads of q and k (of the same tokens) may share memory: their extents within a token, where their tokens step alike, else as a whole."""
    def extent(x, dims):
        return x.data_ptr(), x.data_ptr() + x.element_size() * (1 + sum((x.shape[d] - 1) * x.stride(d) for d in dims))
    if q.numel() == 0 or k.numel() == 0:
        return False
    a, b = extent(q, range(q.dim())), extent(k, range(k.dim()))
    if a[0] >= b[1] or b[0] >= a[1]:
        return False
    if q.dim() == 3 and k.dim() == 3 and q.stride(0) == k.stride(0):
        step = q.stride(0) * q.element_size()
        (q0, q1), (k0, k1) = extent(q, (1, 2)), extent(k, (1, 2))
        low, high = min(q0, k0), max(q1, k1)
        return high - low > step or not (q1 <= k0 or k1 <= q0)
    return True


class PageStep(NamedTuple):
    """What PageTable.extend finds: lengths (requests) with the new tokens, available (1) pages left, starts (requests + 1), slots (tokens, int64; -1: no place),
    positions (tokens), without (1): requests that got no pages."""
    lengths: torch.Tensor
    available: torch.Tensor
    starts: torch.Tensor
    slots: torch.Tensor
    positions: torch.Tensor
    without: torch.Tensor


class PageTable:
    """Pages of a cache's requests, kept on the device.  table: (requests, width) int32, request b's first ceil(lengths[b] / page_size) entries are its pages;
    lengths: (requests) int32;  free: int32, a stack of pages of which the first available[0] are free, taken from its end."""

    def __init__(self, table: torch.Tensor, lengths: torch.Tensor, free: torch.Tensor, available: torch.Tensor, page_size: int):
        if not table.is_cuda:
            raise RuntimeError("table is not a device tensor")
        index = table.get_device()
        if table.dim() != 2 or lengths.shape != table.shape[:1] or free.dim() != 1 or available.shape != (1,) or page_size <= 0:
            raise RuntimeError(f"table {tuple(table.shape)}, lengths {tuple(lengths.shape)}, free {tuple(free.shape)}, available {tuple(available.shape)}, pages of {page_size}")
        for t, name in ((table, "table"), (lengths, "lengths"), (free, "free"), (available, "available")):
            if t.dtype is not torch.int32 or t.get_device() != index or not t.is_contiguous():
                raise RuntimeError(f"{name}: contiguous int32 on {table.device}, not {t.dtype} on {t.device}")
        self._tensors = table, lengths, free, available
        self.page_size, self._index = int(page_size), index
        self._descs = {}
        self._at = lengths.data_ptr(), table.data_ptr(), free.data_ptr(), available.data_ptr()
        self.requests, self.width = table.shape
        if self.width * self.page_size > 0x7FFFFFFF:
            raise RuntimeError(f"{self.width} pages of {self.page_size}: fewer than 2^31 tokens")

    # (not to be replaced: a captured graph holds their addresses)
    table = property(lambda self: self._tensors[0])
    lengths = property(lambda self: self._tensors[1])
    free = property(lambda self: self._tensors[2])
    available = property(lambda self: self._tensors[3])

    @classmethod
    def empty(cls, requests: int, width: int, pages: int, page_size: int, device="cuda:0") -> "PageTable":
        ints = dict(dtype=torch.int32, device=device)
        return cls(torch.full((requests, width), -1, **ints), torch.zeros(requests, **ints), torch.arange(pages - 1, -1, -1, **ints), torch.full((1,), pages, **ints), page_size)

    def _desc(self, tokens):
        return B.PagesDesc(self.requests, self.width, self.page_size, self._tensors[2].shape[0], tokens, self.width)

    def _ints(self, t, name):
        if t.dtype is not torch.int32 or t.shape != (self.requests,) or t.get_device() != self._index:
            raise RuntimeError(f"{name}: int32 ({self.requests}) on {self.table.device}, not {tuple(t.shape)} of {t.dtype} on {t.device}")
        return t if t.is_contiguous() else t.contiguous()

    def extend(self, new: torch.Tensor, tokens: int) -> PageStep:
        """Pages, slots and positions of new[b] tokens of each request b, in a batch of `tokens` rows.  Requests get pages in their order; one whose pages are not all
        there, whose row of the table is full or whose tokens pass the batch gets none.  Entries of new pages are written into the table; lengths and free pages stay as
        they are until the step is accepted (tokens that are only tried need no more)."""
        new = self._ints(new, "new")
        n, tokens = self.requests, int(tokens)
        if tokens < 0:
            raise RuntimeError(f"{tokens} tokens")
        ints = new.new_empty(3 * tokens + 2 * n + 3)                                           # (slots take two each)
        slots, positions, lengths, starts, available, without = ints.split_with_sizes((2 * tokens, tokens, n, n + 1, 1, 1))
        at = ints.data_ptr()
        first = at + 12 * tokens
        desc = self._descs.get(tokens)
        if desc is None:
            if len(self._descs) >= 1024:
                self._descs.clear()
            desc = self._descs[tokens] = self._desc(tokens)
        lengths_at, table_at, free_at, available_at = self._at
        _call(self._index, B.lib.int8t_pages_extend, desc, lengths_at, new.data_ptr(), table_at, free_at, available_at, first, first + 8 * n + 4, first + 4 * n, at, at + 8 * tokens,
              first + 8 * n + 8)
        slots = slots.view(torch.int64)
        return PageStep(lengths, available, starts, slots, positions, without)

    def accept(self, step: PageStep) -> None:
        """The step's tokens and pages become the requests' (no call of this table between its extend and this)."""
        self.lengths.copy_(step.lengths)
        self.available.copy_(step.available)

    def shrink(self, lengths: torch.Tensor) -> None:
        """Requests keep their first lengths[b] tokens (0: ended); pages behind them are free again."""
        stay = self._ints(lengths, "lengths")
        if stay.data_ptr() == self.lengths.data_ptr():
            return
        _call(self._index, B.lib.int8t_pages_shrink, self._desc(0), stay.data_ptr(), self.lengths.data_ptr(), self.table.data_ptr(), self.free.data_ptr(),
              self.available.data_ptr())
