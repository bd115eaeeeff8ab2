"""Token operators (scales per token and output channel, paged cache, attention over it) against plain implementations in 64 bits on the
CPU.  Codes, scales and results that are exact integers scaled in fp32 have to be equal; attention has bounds derived below."""
import math
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import tokens  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


def pad16(n):
    return (n + 15) & ~15


# ---- the definitions, on the CPU (fp32 arithmetic that decides a code evaluated in fp32, the rest in 64 bits) ----------------------
def _mix(x):
    x = np.asarray(x, np.uint64)
    low = np.uint64(0xFFFFFFFF)
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x85EBCA6B)) & low
    x = x ^ (x >> np.uint64(13))
    x = (x * np.uint64(0xC2B2AE35)) & low
    return x ^ (x >> np.uint64(16))


def draws(n, seed):
    low = np.uint64(0xFFFFFFFF)
    lo, hi = np.uint64(seed & 0xFFFFFFFF), np.uint64(seed >> 32)
    kx = _mix(lo ^ _mix((hi + np.uint64(0x9E3779B9)) & low))
    ka = _mix((kx + np.uint64(0x9E3779B9)) & low)
    return _mix(((np.arange(n, dtype=np.uint64) ^ kx) + ka) & low) >> np.uint64(8)


def codes(v, axis, seed=None):
    """Codes (int64) and scales of fp32 v with c the maximum across `axis`."""
    v = np.asarray(v, np.float32)
    c = np.abs(v).max(axis=axis, keepdims=True) if v.size else np.zeros((1, 1), np.float32)
    some = c > 0
    safe = np.where(some, c, np.float32(1))
    inv = np.where(some, np.float32(127) / safe, np.float32(0)).astype(np.float32)
    scale = np.where(some, c / np.float32(127), np.float32(0)).astype(np.float32)
    if seed is None:
        q = np.rint(np.clip(v * inv, np.float32(-127), np.float32(127))).astype(np.int64)
    else:
        u = draws(v.size, seed).reshape(v.shape).astype(np.float64)
        m = np.minimum(np.floor((np.abs(v).astype(np.float64) * (inv.astype(np.float64) * 2.0**24) + u) / 2.0**24), 127)
        q = np.where(v < 0, -m, m).astype(np.int64)
    return q, scale


def scaled(acc, sa, sb=None, bias=None):
    """(float)acc * (sa * sb) + bias, each operation rounded once."""
    s = sa.astype(np.float32) * (np.float32(1) if sb is None else sb.astype(np.float32))
    y = acc.astype(np.float32) * s
    return y if bias is None else y + bias.astype(np.float32)


def values(shape, seed, dtype=F32, spread=1.0):
    r = np.random.default_rng(seed)
    x = r.standard_normal(shape) * np.exp(spread * r.standard_normal(shape[:-1] + (1,)))
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    return t, t.float().numpy()


def unpad(q, cols):
    q = q.cpu().numpy()
    assert not q[:, cols:].any(), "codes beyond the row are not zero"
    return q[:, :cols].astype(np.int64)


def same(got, want, dtype):
    """got (device tensor) equals fp32 `want` rounded once to the type."""
    w = torch.from_numpy(np.ascontiguousarray(want)).to(dtype)
    g = got.detach().cpu()
    assert g.dtype == dtype and g.shape == w.shape
    assert torch.equal(g, w), (g.float() - w.float()).abs().max()


# ---- codes -----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (5, 64), (2, 2048), (3, 2049), (2, 8200), (1, 33001)])
@pytest.mark.parametrize("stochastic,factor", [(False, False), (True, True)])
def test_codes_of_rows(dtype, rows, cols, stochastic, factor):
    x, x32 = values((rows, cols), 1, dtype)
    x[0, 0] = 0.0
    x32[0, 0] = 0.0
    if rows > 2:
        x[1] = 0.0                      # a token of zeros: scale and codes 0
        x32[1] = 0.0
    f = np.random.default_rng(2).random(cols).astype(np.float32) if factor else None
    xd = x.to(DEV)
    q = torch.full((rows, pad16(cols)), 99, dtype=torch.int8, device=DEV)
    s = torch.full((rows,), -1.0, device=DEV)
    fd = None if f is None else torch.from_numpy(f).to(DEV)
    seed = (5 << 40) + 3
    B.int8t_quantize_rows(xd, rows, cols, cols, fd, int(stochastic), seed, q, s, type=B.DTYPES[dtype])
    want, ws = codes(x32 if f is None else x32 * f, 1, seed if stochastic else None)
    assert np.array_equal(unpad(q, cols), want)
    assert np.array_equal(s.cpu().numpy(), ws[:, 0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (17, 3), (130, 70), (1000, 64), (257, 300), (64, 2100)])
@pytest.mark.parametrize("stochastic,factor,sums", [(False, False, False), (True, True, True)])
def test_codes_of_columns(dtype, rows, cols, stochastic, factor, sums):
    x, x32 = values((rows, cols), 3, dtype)
    f = np.random.default_rng(4).random(rows).astype(np.float32) if factor else None
    q = torch.full((cols, pad16(rows)), 99, dtype=torch.int8, device=DEV)
    s = torch.full((cols,), -1.0, device=DEV)
    total = torch.full((cols,), -1.0, device=DEV) if sums else None
    ws = torch.empty(B.int8t_quantize_cols_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    B.int8t_quantize_cols(x.to(DEV), rows, cols, cols, None if f is None else torch.from_numpy(f).to(DEV), int(stochastic), 77, q, s, total, ws,
                          type=B.DTYPES[dtype])
    want, wsc = codes(x32 if f is None else x32 * f[:, None], 0, 77 if stochastic else None)
    assert np.array_equal(unpad(q, rows), want.T)
    assert np.array_equal(s.cpu().numpy(), wsc[0])
    if sums:
        # a lane adds at most rows / 8 values in fp32, eight lanes and the parts follow: fewer than rows + 8 roundings of 2^-24 of the sum of |x|
        x64 = x32.astype(np.float64)
        assert np.all(np.abs(total.cpu().numpy() - x64.sum(0)) <= (rows + 8) * 2.0**-24 * np.abs(x64).sum(0))


@pytest.mark.parametrize("rows,cols", [(1, 1), (16, 16), (100, 33), (129, 65), (300, 1000)])
def test_transposed_codes(rows, cols):
    q = torch.zeros(rows, pad16(cols), dtype=torch.int8)
    q[:, :cols] = torch.from_numpy(np.random.default_rng(5).integers(-127, 128, (rows, cols)).astype(np.int8))
    qt = torch.full((cols, pad16(rows)), 99, dtype=torch.int8, device=DEV)
    B.int8t_transpose_codes(q.to(DEV), rows, cols, qt)
    assert np.array_equal(unpad(qt, rows), q[:, :cols].numpy().astype(np.int64).T)


# ---- products --------------------------------------------------------------------------------------------------------------------
PRODUCTS = [(1, 1, 1), (1, 16, 5), (3, 70, 33), (16, 64, 16), (17, 4096, 1000), (33, 48, 130), (128, 128, 128), (129, 272, 300), (500, 80, 257),
            (64, 9000, 40), (257, 130, 520), (1024, 256, 1040)]


@pytest.mark.parametrize("M,K,N", PRODUCTS)
@pytest.mark.parametrize("dtype,scratch,bias", [(F32, True, True), (BF16, True, False), (F16, False, True)])
def test_product(M, K, N, dtype, scratch, bias):
    r = np.random.default_rng(M + K + N)
    a, b = (r.integers(-127, 128, (n, K)).astype(np.int8) for n in (M, N))
    a[0], b[0] = 127, -127              # the largest sum there is
    sa, sb = (np.exp(r.standard_normal(n)).astype(np.float32) for n in (M, N))
    bv = r.standard_normal(N).astype(np.float32) if bias else None

    def up(c):
        t = torch.zeros(c.shape[0], pad16(K), dtype=torch.int8)
        t[:, :K] = torch.from_numpy(c)
        return t.to(DEV)
    pitch = N + 3
    y = torch.full((M, pitch), 7.0, dtype=dtype, device=DEV)
    ws = torch.empty(max(16, B.int8t_product_workspace_bytes(M, N, K)), dtype=torch.uint8, device=DEV) if scratch else None
    B.int8t_product(up(a), torch.from_numpy(sa).to(DEV), up(b), torch.from_numpy(sb).to(DEV), M, N, K, None if bv is None else torch.from_numpy(bv).to(DEV),
                    y, pitch, type=B.DTYPES[dtype], ws=ws)
    acc = a.astype(np.int64) @ b.astype(np.int64).T
    same(y[:, :N], scaled(acc, sa[:, None], sb[None], bv), dtype)
    assert bool((y[:, N:] == 7.0).all())


@pytest.mark.parametrize("M,K,N", [(1, 300, 40), (2, 4096, 72), (5, 64, 33), (16, 2048, 1000), (31, 130, 64), (70, 512, 96), (300, 1000, 520)])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bias", [False, True])
def test_served_linear(M, K, N, dtype, bias):
    x, x32 = values((M, K), 6, dtype)
    w, w32 = values((N, K), 7, F32, 0.3)
    b = np.random.default_rng(8).standard_normal(N).astype(np.float32) if bias else None
    layer = tokens.ServedLinear.of(w.to(DEV), None if b is None else torch.from_numpy(b).to(DEV))
    wq, sw = codes(w32, 1)
    assert np.array_equal(unpad(layer.codes, K), wq) and np.array_equal(layer.scales.cpu().numpy(), sw[:, 0])
    xq, sx = codes(x32, 1)
    want = scaled(xq @ wq.T, sx, sw.T, b)
    same(layer(x.to(DEV)), want, dtype)
    # rows apart, rows that start off 16 bytes, and leading dimensions
    big = torch.zeros(M, K + 5, dtype=dtype, device=DEV)
    big[:, 3:3 + K] = x.to(DEV)
    same(layer(big[:, 3:3 + K]), want, dtype)
    same(layer(x.to(DEV).view(1, M, K))[0], want, dtype)
    same(layer(x.to(DEV).t().contiguous().t()), want, dtype)


# few tokens: by eight waves, two or one each or two rows of a wave, rows longer than stay in registers, and just too many codes for one launch
@pytest.mark.parametrize("M,K,N", [(1, 9000, 33), (1, 33000, 20), (3, 8200, 40), (4, 20, 17), (7, 4600, 72), (8, 4096, 16), (9, 3600, 40), (13, 2040, 50), (16, 2048, 8200), (16, 2064, 24)])
@pytest.mark.parametrize("dtype", TYPES)
def test_served_few_tokens(M, K, N, dtype):
    test_served_linear(M, K, N, dtype, True)


def _train(x, w, b, g, seed, device=DEV):
    x, w = (t.to(device).requires_grad_(True) for t in (x, w))
    b = None if b is None else torch.from_numpy(b).to(device).requires_grad_(True)
    y = tokens.linear(x, w, b, seed=seed)
    grads = torch.autograd.grad(y, [x, w] + ([] if b is None else [b]), g.to(device))
    return y, grads


@pytest.mark.parametrize("M,K,N", [(1, 16, 16), (2, 33, 5), (70, 130, 65), (256, 512, 1000), (300, 64, 40), (1030, 144, 272)])
@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32)])
def test_linear_and_gradients(M, K, N, dtype, wtype):
    seed = 12345678901234567
    (x, x32), (w, w32), (g, g32) = values((M, K), 9, dtype), values((N, K), 10, wtype, 0.3), values((M, N), 11, dtype)
    b = np.random.default_rng(12).standard_normal(N).astype(np.float32)
    y, (dx, dw, db) = _train(x, w, b, g, seed)
    (xq, sx), (wq, sw) = codes(x32, 1), codes(w32, 1)
    same(y, scaled(xq @ wq.T, sx, sw.T, b), dtype)
    gq, sg = codes(g32 * sw.T, 1, seed)
    same(dx, scaled(gq @ wq, sg), dtype)
    hq, sh = codes(g32 * sx, 0, seed ^ (1 << 63))
    same(dw, scaled(hq.T @ xq, sh.T), wtype)
    g64 = g32.astype(np.float64)
    assert np.all(np.abs(db.cpu().numpy() - g64.sum(0)) <= (M + 8) * 2.0**-24 * np.abs(g64).sum(0) + 1e-30)


# outputs of each length that the gradient's rows are dealt out by, together with its columns up to 8192 and apart beyond
@pytest.mark.parametrize("M,K,N", [(40, 33, 600), (9, 200, 1504), (35, 17, 3001), (130, 48, 8192), (20, 40, 8200), (300, 300, 9001)])
@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_of_wide_outputs(M, K, N, dtype):
    test_linear_and_gradients(M, K, N, dtype, dtype)


def test_gradients_against_differences():
    """Differences of the loss <g, x W^T + b> in 64 bits against the gradients.  dx = sum_n q'[n] wq[n] with q' within one step sg of
    g sw and wq within half a step of w / sw:  |error| <= sum_n sg |wq| + |g sw| / 2; likewise dw over the tokens (|xq| instead)."""
    M, K, N, h = 24, 40, 32, 1e-4
    (x, x32), (w, w32), (g, g32) = values((M, K), 13), values((N, K), 14, F32, 0.3), values((M, N), 15)
    y, (dx, dw, db) = _train(x, w, np.zeros(N, np.float32), g, 5)
    x64, w64, g64 = (t.astype(np.float64) for t in (x32, w32, g32))

    def loss(x, w, b):
        return float((g64 * (x @ w.T + b)).sum())
    (xq, sx), (wq, sw) = codes(x32, 1), codes(w32, 1)
    sg, sh = codes(g32 * sw.T, 1, 5)[1], codes(g32 * sx, 0, 5 ^ (1 << 63))[1]
    bx = sg * np.abs(wq).sum(0) + 0.5 * np.abs(g64 * sw.T).sum(1, keepdims=True)
    bw = sh.T * np.abs(xq).sum(0) + 0.5 * np.abs(g64 * sx).sum(0)[:, None]
    r = np.random.default_rng(16)
    for _ in range(20):
        m, k, n = r.integers(M), r.integers(K), r.integers(N)
        for at, got, bound, arg in (((m, k), dx, bx, 0), ((n, k), dw, bw, 1), ((n,), db, np.full(N, 1e-4), 2)):
            args = [[x64, w64, np.zeros(N)], [x64, w64, np.zeros(N)]]
            for side, sign in ((0, 1), (1, -1)):
                args[side] = [v.copy() for v in args[side]]
                args[side][arg][at] += sign * h
            diff = (loss(*args[0]) - loss(*args[1])) / (2 * h)
            assert abs(float(got[at]) - diff) <= bound[at] * (1 + 1e-6) + 1e-6 * abs(diff) + 1e-6


def test_gradients_are_unbiased():
    """The mean over draws meets the gradient with the same codes of x and W and no rounding of g: a rounded value has variance at most
    (step / 2)^2, so the mean of R draws is within 6 sqrt(sum_n (sg wq / 2)^2 / R) for all but one in 5e8 elements."""
    M, K, N, R = 6, 48, 40, 256
    (x, x32), (w, w32), (g, g32) = values((M, K), 17), values((N, K), 18, F32, 0.3), values((M, N), 19)
    (xq, sx), (wq, sw) = codes(x32, 1), codes(w32, 1)
    mx, mw = torch.zeros(M, K, dtype=torch.float64, device=DEV), torch.zeros(N, K, dtype=torch.float64, device=DEV)
    for seed in range(R):
        _, (dx, dw) = _train(x, w, None, g, seed)
        mx += dx.double() / R
        mw += dw.double() / R
    a, b = g32 * sw.T, g32 * sx
    sg, sh = codes(a, 1, 0)[1], codes(b, 0, 0)[1]
    for got, want, var in ((mx, a.astype(np.float64) @ wq, (sg / 2) ** 2 * (wq.astype(np.float64) ** 2).sum(0)),
                           (mw, b.astype(np.float64).T @ xq, (sh.T / 2) ** 2 * (xq.astype(np.float64) ** 2).sum(0))):
        assert np.all(np.abs(got.cpu().numpy() - want) <= 6 * np.sqrt(var / R) + 1e-6)


def test_linear_of_no_tokens_and_single_gradients():
    x, w = torch.zeros(0, 48, device=DEV, requires_grad=True), torch.randn(20, 48, device=DEV, requires_grad=True)
    b = torch.zeros(20, device=DEV, requires_grad=True)
    y = tokens.linear(x, w, b)
    assert y.shape == (0, 20)
    dx, dw, db = torch.autograd.grad(y, [x, w, b], torch.zeros(0, 20, device=DEV))
    assert dx.shape == (0, 48) and not dw.any() and not db.any()
    assert tokens.ServedLinear.of(w)(torch.zeros(2, 0, 48, device=DEV)).shape == (2, 0, 20)
    # one gradient at a time gives what all together give; a gradient that is broadcast (strides of 0) is one like any other
    x, g = torch.randn(33, 48, device=DEV), torch.randn(33, 20, device=DEV)
    xs, ws, bs = x.requires_grad_(True), w, b
    everything = torch.autograd.grad(tokens.linear(xs, ws, bs, seed=4), [xs, ws, bs], g)
    assert torch.equal(torch.autograd.grad(tokens.linear(xs, ws.detach(), None, seed=4), xs, g)[0], everything[0])
    assert torch.equal(torch.autograd.grad(tokens.linear(xs.detach(), ws, None, seed=4), ws, g)[0], everything[1])
    only = torch.autograd.grad(tokens.linear(xs.detach(), ws.detach(), bs, seed=4), bs, g)[0]
    assert torch.allclose(only, everything[2], rtol=1e-5, atol=1e-5)
    row = torch.randn(20, device=DEV)
    a = torch.autograd.grad(tokens.linear(xs, ws, bs, seed=4), [xs, ws], row.expand(33, 20))
    c = torch.autograd.grad(tokens.linear(xs, ws, bs, seed=4), [xs, ws], row.repeat(33, 1))
    assert all(torch.equal(p, q) for p, q in zip(a, c))


def test_token_linear_module():
    m = tokens.TokenLinear(64, 40, dtype=BF16, name="proj", device=DEV)
    x = torch.randn(3, 5, 64, dtype=BF16, device=DEV)
    y = m(x)
    y.float().square().sum().backward()
    assert m.weight.grad.dtype is BF16 and m.weight.grad.shape == (40, 64) and m.bias.grad.dtype is F32
    assert torch.equal(m.served()(x), y.detach())
    seed = m._seed
    with torch.no_grad():
        assert torch.equal(m(x), y)
    assert m._seed == seed


# ---- cache -----------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens_,heads,dim,page", [(1, 1, 16, 1), (7, 3, 64, 16), (33, 2, 80, 24), (19, 5, 128, 7), (40, 12, 256, 64), (300, 8, 96, 32)])
def test_cache_write_and_read(dtype, tokens_, heads, dim, page):
    pages = -(-2 * tokens_ // page) + 1
    cache = tokens.PagedCache.empty(pages, page, heads, dim, DEV)
    for t in (cache.kq, cache.vq):
        t.fill_(3)
    for t in (cache.ks, cache.vs):
        t.fill_(0.5)
    (k, k32), (v, v32) = values((tokens_, heads, dim), 21, dtype), values((tokens_, heads, dim), 22, dtype)
    k[0, 0], k32[0, 0] = 0.0, 0.0
    r = np.random.default_rng(23)
    slots = r.permutation(pages * page)[:tokens_].astype(np.int64)
    if tokens_ > 4:
        slots[2], slots[4] = -1, pages * page + 5         # left out
    # keys and values as parts of one projection, off 16 bytes
    both = torch.zeros(tokens_, 2 * heads * dim + 1, dtype=dtype, device=DEV)
    both[:, 1:1 + heads * dim] = k.view(tokens_, -1).to(DEV)
    both[:, 1 + heads * dim:] = v.view(tokens_, -1).to(DEV)
    cache.write(both[:, 1:1 + heads * dim].view(tokens_, heads, dim), both[:, 1 + heads * dim:].view(tokens_, heads, dim), torch.from_numpy(slots).to(DEV))
    want = {}
    for name, x in (("k", k32), ("v", v32)):
        q, s = np.full((pages, heads, page, dim), 3, np.int64), np.full((pages, heads, page), 0.5, np.float32)
        c, sc = codes(x, 2)
        for t, at in enumerate(slots):
            if 0 <= at < pages * page:
                q[at // page, :, at % page], s[at // page, :, at % page] = c[t], sc[t, :, 0]
        want[name] = q, s
    for name in ("k", "v"):
        assert np.array_equal(getattr(cache, name + "q").cpu().numpy(), want[name][0])
        assert np.array_equal(getattr(cache, name + "s").cpu().numpy(), want[name][1])
    back = np.concatenate([slots, r.integers(0, pages * page, 5)])
    got = cache.read(torch.from_numpy(back).to(DEV), dtype)
    for name, t in zip("kv", got):
        q, s = want[name]
        ref = np.stack([q[a // page, :, a % page].astype(np.float32) * s[a // page, :, a % page, None] if 0 <= a < pages * page
                        else np.zeros((heads, dim), np.float32) for a in back])
        same(t, ref, dtype)


def test_cache_of_aligned_rows_and_no_tokens():
    cache = tokens.PagedCache.empty(4, 16, 2, 64, DEV)
    k, v = (torch.randn(9, 2, 64, device=DEV) for _ in range(2))
    slots = torch.arange(9, device=DEV) * 5
    cache.write(k, v, slots)
    c, s = codes(k.cpu().numpy(), 2)
    same(cache.read(slots)[0], c.astype(np.float32) * s, F32)
    before = cache.kq.clone()
    cache.write(k[:0], v[:0], slots[:0])
    assert torch.equal(cache.kq, before) and cache.read(slots[:0])[0].shape == (0, 2, 64)
    # heads first in memory
    cache.write(k.transpose(0, 1).contiguous().transpose(0, 1), v, slots)
    assert torch.equal(cache.kq, before)


# ---- attention -------------------------------------------------------------------------------------------------------------------
def attend_reference(cache, q, starts, lengths, table, causal, scale):
    """64 bits: (output, sum of p |v| / sum of p, logarithm of the sum, largest |scale ks sum |q kq|| of a row)."""
    kq, ks, vq, vs = (t.cpu().double() for t in (cache.kq, cache.ks, cache.vq, cache.vs))
    T, HQ, D = q.shape
    H, page = cache.heads, cache.page_size
    G = HQ // H
    out, absolute = torch.zeros(T, HQ, D, dtype=torch.float64), torch.zeros(T, HQ, D, dtype=torch.float64)
    lse, size = torch.full((T, HQ), -math.inf, dtype=torch.float64), torch.zeros(T, HQ, dtype=torch.float64)
    q = q.cpu().double()
    for b in range(len(lengths)):
        n, L = starts[b + 1] - starts[b], lengths[b]
        for i in range(n):
            end = min(L, L - n + i + 1) if causal else L
            js = [j for j in range(max(0, end)) if 0 <= table[b][j // page] < cache.pages]
            if not js:
                continue
            p_ids, o_ids = torch.tensor([table[b][j // page] for j in js]), torch.tensor([j % page for j in js])
            for hq in range(HQ):
                h = hq // G
                k = kq[p_ids, h, o_ids] * ks[p_ids, h, o_ids][:, None]
                v = vq[p_ids, h, o_ids] * vs[p_ids, h, o_ids][:, None]
                t = starts[b] + i
                s = k @ q[t, hq] * scale
                p = torch.exp(s - s.max())
                out[t, hq], absolute[t, hq] = p @ v / p.sum(), p @ v.abs() / p.sum()
                lse[t, hq] = s.max() + torch.log(p.sum())
                size[t, hq] = (k.abs() @ q[t, hq].abs()).max() * abs(scale)
    return out, absolute, lse, size


def check_attend(cache, q, starts, lengths, table, causal=True, scale=None, longest=None, poison=True):
    """Runs and compares.  Bound of an element: scores carry errors of their fp32 sums, of the pieces of q (fp32: 22 bits; otherwise exact)
    and of the exponential's argument, together under ds = 2^-18 of the sum of |terms| + 2^-20; p is rounded to 11 bits (fp32: 22),
    the output to its type:  (2 ds + e_p) * (sum p |v| / sum p) + e_out |o|.  p vs is held in fp16 times 2^15 / (largest vs), a fixed point
    with steps of 2^-24 where it is small: 2^-40 of the largest value, 127 vs, for each key."""
    dt = q.dtype
    e_p, e_out = {F32: (2.0**-20, 2.0**-22), BF16: (2.0**-10.9, 2.0**-8), F16: (2.0**-10.9, 2.0**-10.9)}[dt]
    scale_ = 1 / math.sqrt(cache.dim) if scale is None else scale
    want, absolute, lse, size = attend_reference(cache, q, starts, lengths, table, causal, scale_)
    width = max(1, max(len(t) for t in table)) if table else 1
    t = torch.full((len(table), width), 0x7FFFFFF0, dtype=torch.int32)       # (what no length needs is not looked at)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, lengths)]
    got, glse = cache.attend(q, args[0], args[1], t.to(DEV), causal=causal, scale=scale, longest=longest, return_lse=True)
    assert got.dtype == dt and got.shape == q.shape
    got, glse = got.cpu().double(), glse.cpu().double()
    ds = 2.0**-18 * size + 2.0**-20
    used = cache.vs[torch.isfinite(cache.vs)]
    floor = max(lengths) * 127 * 2.0**-40 * float(used.max()) if used.numel() else 0.0
    bound = (2 * ds[..., None] + e_p) * absolute + e_out * want.abs() + floor + 1e-30
    if dt is F16:
        bound = bound + 2.0**-25                                            # (smallest fp16 step, halved)
    assert bool(((got - want).abs() <= bound).all()), ((got - want).abs() / bound).max()
    none = torch.isinf(lse)
    assert torch.equal(none, torch.isinf(glse) & (glse < 0)) and not got[none].any()
    assert bool(((glse - lse)[~none].abs() <= 2 * ds[~none] + 2.0**-20 * lse[~none].abs() + 2.0**-18).all())
    return got


def make_cache(lengths, heads, dim, page, seed=0, extra=2, poison=True):
    """A cache with the pages of requests of those lengths in random order; what no request uses holds NaN scales."""
    r = np.random.default_rng(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + extra
    ids = r.permutation(pages).tolist()
    table = [[ids.pop() for _ in range(n)] for n in need]
    gen = torch.Generator().manual_seed(seed)
    q = [torch.randint(-127, 128, (pages, heads, page, dim), generator=gen, dtype=torch.int8) for _ in range(2)]
    s = [torch.exp(0.5 * torch.randn(pages, heads, page, generator=gen)) / 64 for _ in range(2)]
    if poison:
        used = torch.zeros(pages, page, dtype=torch.bool)
        for row, n in zip(table, lengths):
            for j in range(n):
                used[row[j // page], j % page] = True
        for t in s:
            t[~used[:, None].expand(pages, heads, page)] = float("nan")
    return tokens.PagedCache(q[0].to(DEV), s[0].to(DEV), q[1].to(DEV), s[1].to(DEV)), table


def queries(T, heads, dim, dtype, seed=1):
    return (torch.randn(T, heads, dim, generator=torch.Generator().manual_seed(seed)) * 1.5).to(dtype).to(DEV)


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)]).tolist()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,dim,page", [(1, 1, 16, 1), (2, 4, 64, 16), (3, 7, 80, 24), (2, 1, 96, 5), (2, 8, 128, 16), (1, 16, 128, 64), (1, 3, 256, 32),
                                                  (2, 20, 48, 8)])
def test_attend_single_tokens(dtype, heads, group, dim, page):
    lengths = [1, 33, 0, 257, 31, 500]
    cache, table = make_cache(lengths, heads, dim, page)
    check_attend(cache, queries(len(lengths), heads * group, dim, dtype), starts_of([1] * len(lengths)), lengths, table)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim,page", [(2, 4, 64, 16), (1, 3, 80, 24), (2, 1, 128, 7), (1, 2, 256, 32), (1, 8, 128, 64)])
def test_attend_chunks(dtype, causal, heads, group, dim, page):
    new, lengths = [17, 0, 1, 70, 5], [17, 9, 40, 200, 131]
    cache, table = make_cache(lengths, heads, dim, page)
    check_attend(cache, queries(sum(new), heads * group, dim, dtype), starts_of(new), lengths, table, causal=causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("new", [40, 300])
def test_attend_rows_that_see_nothing(dtype, new):
    """More new tokens than keys (causal): the first see nothing; a request without keys; one whose pages are not in the cache."""
    lengths = [11, 0, 64]
    cache, table = make_cache(lengths, 2, 64, 16)
    table[2] = [cache.pages + 3, -1, table[2][2], 1 << 30]
    got = check_attend(cache, queries(3 * new, 4, 64, dtype), starts_of([new] * 3), lengths, table)
    assert not got[:new - 11].any() and not got[new:2 * new].any()


@pytest.mark.parametrize("dtype,heads,group,dim,page,new,lengths", [
    (BF16, 2, 4, 128, 64, [1024, 700], [4096, 3001]), (F16, 2, 2, 64, 16, [900, 1500], [2500, 1500]), (F32, 1, 4, 128, 24, [600, 64], [2100, 3000]),
    (BF16, 1, 8, 256, 32, [300, 90], [3000, 1111]), (F16, 1, 16, 128, 16, [1] * 40, list(range(7, 6000, 150)))])
def test_attend_of_many_tiles(dtype, heads, group, dim, page, new, lengths):
    """Hundreds of tiles of keys and several blocks, against 64 bits on the GPU; bounds as in check_attend(), the keys' spread from its definition."""
    cache, table = make_cache(lengths, heads, dim, page, poison=False)
    q = queries(sum(new), heads * group, dim, dtype)
    t = torch.zeros(len(new), max(map(len, table)), dtype=torch.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row)
    starts = starts_of(new)
    args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, lengths)]
    got = cache.attend(q, args[0], args[1], t.to(DEV), longest=max(lengths)).double()
    e_p, e_out = {F32: (2.0**-20, 2.0**-22), BF16: (2.0**-10.9, 2.0**-8), F16: (2.0**-10.9, 2.0**-10.9)}[dtype]
    for b, (n, L) in enumerate(zip(new, lengths)):
        ids = torch.tensor(table[b], device=DEV)
        k, v = ((c[ids].double() * s[ids].double()[..., None]).transpose(0, 1).reshape(heads, -1, dim)[:, :L] for c, s in ((cache.kq, cache.ks), (cache.vq, cache.vs)))
        rows = q[starts[b]:starts[b + 1]].double().view(n, heads, group, dim)
        last = L - n + torch.arange(n, device=DEV)
        for h in range(heads):
            for g in range(group):
                a = rows[:, h, g] @ k[h].t() / math.sqrt(dim)
                size = (rows[:, h, g].abs() @ k[h].abs().t()).amax(1) / math.sqrt(dim)
                a = a.masked_fill(torch.arange(L, device=DEV) > last[:, None], -math.inf)
                p = torch.softmax(a, 1)
                want, absolute = p @ v[h], p @ v[h].abs()
                bound = (2 * (2.0**-18 * size[:, None] + 2.0**-20) + e_p) * absolute + e_out * want.abs() + L * 127 * 2.0**-40 * cache.vs.max().double() + 2.0**-25
                off = (got[starts[b]:starts[b + 1], h * group + g] - want).abs() / bound
                assert float(off.max()) <= 1, (b, h, g, float(off.max()))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,heads,group,dim,page,new,lengths", [
    (BF16, 2, 4, 128, 7, [40, 33, 90], [41, 500, 1300]), (F16, 1, 8, 96, 24, [17, 70], [300, 129]), (F32, 1, 4, 128, 24, [700, 600], [700, 1500]),
    (F32, 1, 4, 112, 32, [513, 700], [2000, 611]), (F32, 2, 4, 64, 7, [130, 90], [130, 400]), (BF16, 1, 3, 48, 24, [90, 50], [77, 301]),
    (F32, 1, 8, 256, 5, [60, 40], [200, 65]), (F16, 1, 3, 144, 16, [80, 55], [1000, 55])])
def test_attend_of_larger_blocks(dtype, causal, heads, group, dim, page, new, lengths):
    """Enough rows of a request for blocks of 128 or 256 rows, ragged; pages that end inside a tile and dims that end inside a block's."""
    cache, table = make_cache(lengths, heads, dim, page)
    q = queries(sum(new), heads * group, dim, dtype)
    t = torch.full((len(new), max(map(len, table))), 0x7FFFFFF0, dtype=torch.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row)
    starts = starts_of(new)
    args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, lengths)]
    got, glse = cache.attend(q, args[0], args[1], t.to(DEV), causal=causal, return_lse=True)
    got, glse = got.double(), glse.double()
    e_p, e_out = {F32: (2.0**-20, 2.0**-22), BF16: (2.0**-10.9, 2.0**-8), F16: (2.0**-10.9, 2.0**-10.9)}[dtype]
    for b, (n, L) in enumerate(zip(new, lengths)):
        ids = torch.tensor(table[b], device=DEV)
        k, v = ((c[ids].double() * s[ids].double()[..., None]).transpose(0, 1).reshape(heads, -1, dim)[:, :L] for c, s in ((cache.kq, cache.ks), (cache.vq, cache.vs)))
        largest = float(torch.where(torch.isfinite(cache.vs), cache.vs, torch.zeros_like(cache.vs)).max())
        rows = q[starts[b]:starts[b + 1]].double().view(n, heads, group, dim)
        seen = torch.arange(L, device=DEV) <= (L - n + torch.arange(n, device=DEV))[:, None] if causal else torch.ones(n, L, dtype=torch.bool, device=DEV)
        none = ~seen.any(1)
        for h in range(heads):
            for g in range(group):
                at = slice(starts[b], starts[b + 1]), h * group + g
                a = rows[:, h, g] @ k[h].t() / math.sqrt(dim)
                size = (rows[:, h, g].abs() @ k[h].abs().t()).amax(1) / math.sqrt(dim)
                a = a.masked_fill(~seen, -math.inf)
                p = torch.nan_to_num(torch.softmax(a, 1))
                want, absolute = p @ v[h], p @ v[h].abs()
                ds = 2.0**-18 * size + 2.0**-20
                bound = (2 * ds[:, None] + e_p) * absolute + e_out * want.abs() + L * 127 * 2.0**-40 * largest + 2.0**-25
                assert float(((got[at] - want).abs() / bound).max()) <= 1, (b, h, g)
                assert not got[at][none].any() and bool((glse[at][none] == -math.inf).all())
                lse = torch.logsumexp(a[~none], 1)
                assert bool(((glse[at][~none] - lse).abs() <= 2 * ds[~none] + 2.0**-20 * lse.abs() + 2.0**-18).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_attend_long_context(dtype):
    lengths = [16001, 3, 8000]
    cache, table = make_cache(lengths, 1, 128, 16, poison=False)
    check_attend(cache, queries(5, 4, 128, dtype), starts_of([1, 1, 3]), lengths, table)
    check_attend(cache, queries(5, 4, 128, dtype), starts_of([1, 1, 3]), lengths, table, longest=16001)
    check_attend(cache, queries(5, 4, 128, dtype), starts_of([1, 1, 3]), lengths, table, longest=1)      # (a guide only)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[1, 1], [40, 90]])
def test_attend_scales_far_apart(dtype, new):
    """Scores of hundreds, value scales over twelve orders of magnitude, queries from 1e-20 to 1e4: the running maximum and the reference
    of the value scales move often.  fp16's own p keeps an absolute 2^-25 of the largest scale seen, which the bound allows for."""
    lengths = [150, 333]
    cache, table = make_cache(lengths, 1, 64, 16, seed=4)
    cache.ks.mul_(torch.exp(2 * torch.randn(cache.ks.shape, generator=torch.Generator().manual_seed(5))).to(DEV))
    q = queries(sum(new), 2, 64, F32)
    q = (q * torch.logspace(-4, 1, q.shape[0] * 2, device=DEV).view(-1, 2, 1)).to(dtype)
    q[0] *= 0.0
    check_attend(cache, q, starts_of(new), lengths, table)
    # value scales: compared with the row's largest value, not with its own sum
    cache.vs.mul_(torch.logspace(-6, 6, cache.vs.shape[0], device=DEV)[:, None, None])
    want, _, _, _ = attend_reference(cache, q, starts_of(new), lengths, table, True, 1 / 8)
    tt = torch.zeros(2, max(map(len, table)), dtype=torch.int32)
    for b, row in enumerate(table):
        tt[b, :len(row)] = torch.tensor(row)
    got = cache.attend(q, torch.tensor(starts_of(new), dtype=torch.int32, device=DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), tt.to(DEV)).cpu().double()
    largest = 127 * float(cache.vs[torch.isfinite(cache.vs)].max())
    if dtype is not F16:
        assert bool(((got - want).abs() <= 2.0**-8 * want.abs() + 2.0**-9 * largest * 1e-3 + 2e-3 * want.abs().max()).all())


def test_attend_strided_queries_and_repeats():
    lengths, new = [70, 45], [9, 33]
    cache, table = make_cache(lengths, 2, 64, 16)
    fused = torch.randn(42, 3, 8, 64, device=DEV, dtype=BF16)
    q = fused[:, 1]
    a = check_attend(cache, q, starts_of(new), lengths, table)
    off = torch.zeros(42 * 8 * 64 + 1, device=DEV, dtype=BF16)
    off[1:] = q.reshape(-1)
    assert torch.equal(check_attend(cache, off[1:].view(42, 8, 64), starts_of(new), lengths, table), a)
    assert torch.equal(check_attend(cache, q.transpose(0, 1).contiguous().transpose(0, 1), starts_of(new), lengths, table), a)
    for _ in range(3):
        assert torch.equal(check_attend(cache, q.contiguous(), starts_of(new), lengths, table), a)


def test_attend_rows_do_not_touch_each_other():
    lengths, new = [90, 50], [20, 4]
    cache, table = make_cache(lengths, 1, 64, 16)
    q = queries(24, 2, 64, F32)
    clean = check_attend(cache, q, starts_of(new), lengths, table)
    q[5, 1, 7], q[21, 0, 3] = float("nan"), float("inf")
    t = torch.zeros(2, 6, dtype=torch.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row)
    got = cache.attend(q, torch.tensor(starts_of(new), dtype=torch.int32, device=DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), t.to(DEV)).cpu().double()
    same_rows = torch.ones(24, 2, dtype=torch.bool)
    same_rows[5, 1] = same_rows[21, 0] = False
    assert torch.equal(got[same_rows], clean[same_rows])


def test_cache_beyond_four_gib():
    """Places whose codes lie past 2^32 bytes."""
    pages, page, heads, dim = 70000, 32, 8, 256
    if torch.cuda.mem_get_info()[0] < 16 << 30:
        pytest.skip("needs 16 GiB")
    assert pages * page * heads * dim > 1 << 32
    q = [torch.empty(pages, heads, page, dim, dtype=torch.int8, device=DEV) for _ in range(2)]
    s = [torch.zeros(pages, heads, page, device=DEV) for _ in range(2)]
    cache = tokens.PagedCache(q[0], s[0], q[1], s[1])
    rows = [[pages - 1, 0], [pages - 2, pages // 2]]
    lengths = [50, 64]
    k, v = (torch.randn(114, heads, dim, device=DEV) for _ in range(2))
    slots = torch.tensor([rows[b][j // page] * page + j % page for b in range(2) for j in range(lengths[b])], device=DEV)
    cache.write(k, v, slots)
    c, sc = codes(k.cpu().numpy(), 2)
    same(cache.read(slots)[0], c.astype(np.float32) * sc, F32)
    # the same tokens in a small cache
    small = tokens.PagedCache.empty(4, page, heads, dim, DEV)
    near = torch.tensor([(2 * b + j // page) * page + j % page for b in range(2) for j in range(lengths[b])], device=DEV)
    small.write(k, v, near)
    qq = queries(2, heads * 2, dim, F32)
    starts, le = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, 1, 2], lengths))
    a = cache.attend(qq, starts, le, torch.tensor(rows, dtype=torch.int32, device=DEV))
    b = small.attend(qq, starts, le, torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device=DEV))
    assert torch.equal(a, b)


# ---- streams, graphs -------------------------------------------------------------------------------------------------------------
def _pass(layer, cache, x, slots, starts, lengths, table):
    y = layer(x)
    q, k, v = y.split([256, 128, 128], dim=1)
    cache.write(k.view(-1, 2, 64), v.view(-1, 2, 64), slots)
    return cache.attend(q.view(-1, 4, 64), starts, lengths, table)


def test_another_stream_and_graph_replays():
    layer = tokens.ServedLinear.of(torch.randn(512, 96, device=DEV) * 0.1)
    x = torch.randn(3, 96, device=DEV, dtype=BF16)
    lengths0 = [40, 21, 65]
    cache, table = make_cache([80, 80, 80], 2, 64, 16, poison=False)
    t = torch.tensor(table, dtype=torch.int32, device=DEV)
    starts = torch.arange(4, dtype=torch.int32, device=DEV)
    lengths = torch.tensor(lengths0, dtype=torch.int32, device=DEV)

    def slots_of(ls):
        return torch.tensor([table[b][(n - 1) // 16] * 16 + (n - 1) % 16 for b, n in enumerate(ls)], device=DEV)
    slots = slots_of(lengths0)
    want = _pass(layer, cache, x, slots, starts, lengths, t).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _pass(layer, cache, x, slots, starts, lengths, t)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _pass(layer, cache, x, slots, starts, lengths, t)
    for step in range(4):
        ls = [n + step for n in lengths0]
        x.copy_(torch.randn(3, 96, generator=torch.Generator().manual_seed(step)))
        lengths.copy_(torch.tensor(ls, dtype=torch.int32))
        slots.copy_(slots_of(ls))
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(replayed, _pass(layer, cache, x, slots, starts, lengths, t))


# ---- refusals --------------------------------------------------------------------------------------------------------------------
def test_refusals():
    layer = tokens.ServedLinear.of(torch.randn(8, 32, device=DEV))
    cache = tokens.PagedCache.empty(2, 16, 2, 64, DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    s, n, t = torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros(1, 2, **i32)
    q = torch.zeros(1, 4, 64, device=DEV)
    k = torch.zeros(3, 2, 64, device=DEV)
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    for call in (lambda: layer(torch.zeros(2, 31, device=DEV)), lambda: layer(torch.zeros(2, 32)), lambda: tokens.linear(torch.zeros(2, 32, device=DEV), torch.zeros(4, 31, device=DEV)),
                 lambda: tokens.linear(torch.zeros(2, 32, device=DEV), torch.zeros(4, 32, device=DEV), torch.zeros(5, device=DEV)),
                 lambda: tokens.linear(torch.zeros(2, 32, device=DEV), torch.zeros(4, 32, device=DEV), torch.zeros(4, device=DEV, dtype=BF16)),
                 lambda: cache.write(k, k, slots[:2]), lambda: cache.write(k, k[:2], slots), lambda: cache.write(k.bfloat16(), k, slots), lambda: cache.write(k, k, slots.int()),
                 lambda: cache.read(slots.cpu()), lambda: cache.attend(q[..., :32], s, n, t), lambda: cache.attend(torch.zeros(1, 3, 64, device=DEV), s, n, t),
                 lambda: cache.attend(q, s.long(), n, t), lambda: cache.attend(q, s[:1], n, t), lambda: cache.attend(q, s, n, t[0]), lambda: cache.attend(q.cpu(), s, n, t),
                 lambda: tokens.PagedCache.empty(2, 16, 2, 60, DEV), lambda: tokens.PagedCache.empty(2, 16, 2, 272, DEV),
                 lambda: tokens.ServedLinear(layer.codes, layer.scales[:4], 32), lambda: tokens.ServedLinear(layer.codes, layer.scales, 33)):
        with pytest.raises(RuntimeError):
            call()
    for call in (lambda: layer(torch.zeros(2, 32, device=DEV, dtype=torch.float64)), lambda: cache.read(slots, torch.float64), lambda: cache.write(k.double(), k.double(), slots)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(B.Int8tError) as e:          # a reduction whose sums may not fit
        tokens.ServedLinear(torch.zeros(1, 131088, dtype=torch.int8, device=DEV), torch.ones(1, device=DEV), 131088)(torch.zeros(1, 131088, device=DEV))
    assert e.value.status == 2
