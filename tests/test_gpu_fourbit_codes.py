"""Microscaled 4-bit codes of matrices, along rows and columns, and products of them, against plain implementations in 64 bits.  Codes and scales have to be equal."""
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

import fourbit_reference as R  # noqa: E402
from paper_1912_12607_amd import binding as B  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


def values(shape, seed, dtype=F32, spread=1.5):
    r = np.random.default_rng(seed)
    x = r.standard_normal(shape) * np.exp(spread * r.standard_normal(shape[:-1] + (1,)))
    t = torch.from_numpy(x.astype(np.float32)).to(dtype)
    return t, t.double().numpy()


def quantise(xd, rows, cols, pitch, dtype, stochastic=False, seed=0, q=True, qt=True, sums=True):
    """(codes, scales) by rows and by columns (each as the reference has them), sums; room behind every output is checked."""
    def room(n):
        return torch.full((n + 64,), 0x5A, dtype=torch.uint8, device=DEV)
    nq, ns = rows * 16 * R.blocks_of(cols), R.panels_of(cols) * rows * 8
    nqt, nst = cols * 16 * R.blocks_of(rows), R.panels_of(rows) * cols * 8
    bufs = [room(n) for n in (nq, ns, nqt, nst)]
    total = torch.full((cols + 1,), 7.0, device=DEV)
    ws = torch.empty(B.int8t_mx4_quantize_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    B.int8t_mx4_quantize(xd, rows, cols, pitch, int(stochastic), seed, bufs[0] if q else None, bufs[1] if q else None, bufs[2] if qt else None,
                         bufs[3] if qt else None, total if sums else None, ws if sums else None, type=B.DTYPES[dtype])
    out = []
    for used, code, scale, nc, nsc, r, c in ((q, bufs[0], bufs[1], nq, ns, rows, cols), (qt, bufs[2], bufs[3], nqt, nst, cols, rows)):
        code, scale = code.cpu().numpy(), scale.cpu().numpy()
        assert (code[nc if used else 0:] == 0x5A).all() and (scale[nsc if used else 0:] == 0x5A).all()
        out.append((code[:nc].reshape(r, -1), scale[:nsc].reshape(-1, r, 8)) if used else None)
    t = total.cpu().numpy()
    assert t[cols] == 7.0 and (sums or (t == 7.0).all())
    return out[0], out[1], t[:cols]


def check(got, x, cols, u=None):
    code, byte = R.quantise(x, u)
    assert np.array_equal(got[1], R.in_panels(byte, cols))
    assert np.array_equal(got[0], R.packed(code))


SIZES = [(1, 1), (1, 32), (3, 7), (5, 64), (33, 31), (32, 33), (2, 2048), (255, 257), (257, 300), (64, 2100), (1000, 40), (1, 33001), (33001, 2)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("stochastic", [False, True])
def test_codes(dtype, rows, cols, stochastic):
    x, x64 = values((rows, cols), rows + cols, dtype)
    if rows > 2:
        x[1], x64[1] = 0.0, 0.0                     # a token of zeros
    seed = (5 << 40) + 3
    by_rows, by_cols, sums = quantise(x.to(DEV), rows, cols, cols, dtype, stochastic, seed)
    index = np.arange(rows * cols).reshape(rows, cols)
    check(by_rows, x64, cols, R.draws(index, seed) if stochastic else None)
    check(by_cols, x64.T, rows, R.draws(index, seed ^ (1 << 63)).T if stochastic else None)
    # sums of 32 values in fp32 (32 roundings), of the blocks in 64 bits, one rounding
    assert (np.abs(sums - x64.sum(0)) <= 33 * 2.0**-24 * np.abs(x64).sum(0)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_of_strided_rows_and_single_outputs(dtype):
    rows, cols, pitch = 70, 90, 101
    x, _ = values((rows, pitch + 3), 4, dtype)
    at = x.reshape(-1)[3:3 + rows * pitch].reshape(rows, pitch)          # off 16 bytes too
    xd = at.to(DEV)
    x64 = at[:, :cols].double().numpy()
    for q, qt, sums in ((True, False, False), (False, True, False), (False, False, True), (True, True, False)):
        by_rows, by_cols, s = quantise(xd, rows, cols, pitch, dtype, q=q, qt=qt, sums=sums)
        if q:
            check(by_rows, x64, cols)
        if qt:
            check(by_cols, x64.T, rows)
        if sums:
            assert (np.abs(s - x64.sum(0)) <= 33 * 2.0**-24 * np.abs(x64).sum(0)).all()


def test_codes_at_ties_borders_and_the_ends_of_the_range():
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    near = np.concatenate([ties, np.nextafter(ties.astype(np.float32), np.float32(0)), np.nextafter(ties[:7].astype(np.float32), np.float32(9)), [0.0, 1e-30, 1e-45]])
    rows = []
    for e in (-149, -148, -130, -127, -126, -125, -20, -1, 0, 1, 60, 124, 125):
        row = np.zeros(64, np.float32)
        with np.errstate(all="ignore"):
            row[:len(near)] = np.ldexp(near, e).astype(np.float32)
            row[32:64] = -row[:32]
            # the largest of a block at its border: 6 2^e exactly, and the next value
            row[40] = np.float32(np.ldexp(6.0, min(e, 125)))
        rows.append(row)
        up = row.copy()
        up[5] = np.nextafter(np.float32(np.ldexp(6.0, min(e, 125))), np.float32(np.inf))
        rows.append(up)
    rows.append(np.full(64, np.finfo(np.float32).max, np.float32))
    rows.append(np.full(64, 1e-45, np.float32))
    x = np.stack(rows)
    by_rows, by_cols, _ = quantise(torch.from_numpy(x).to(DEV), *x.shape, 64, F32, sums=False)
    check(by_rows, x, 64)
    check(by_cols, x.T, x.shape[0])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_codes_of_what_is_not_finite(dtype, stochastic, bad):
    x, _ = values((70, 80), 9, dtype)
    x[3, 40] = x[40, 79] = bad
    x64 = x.double().numpy()
    by_rows, by_cols, _ = quantise(x.to(DEV), 70, 80, 80, dtype, stochastic, 11, sums=False)
    index = np.arange(70 * 80).reshape(70, 80)
    check(by_rows, x64, 80, R.draws(index, 11) if stochastic else None)
    check(by_cols, x64.T, 70, R.draws(index, 11 ^ (1 << 63)).T if stochastic else None)
    assert by_rows[1][0, 3, 1] == 255 and by_rows[1][0, 3, 0] < 255


def test_stochastic_codes_are_unbiased():
    x = torch.linspace(-6, 6, 64, device=DEV).repeat(4096, 1) * 0.37
    by_rows, _, _ = quantise(x, 4096, 64, 64, F32, True, 5, qt=False, sums=False)
    byte = by_rows[1][0, :, :2]
    mean = R.stands_for(R.unpacked(by_rows[0]), byte, 64).mean(0)
    # a step is at most 2 2^e (2^e < 1/2 here); the mean of 4096 draws is off by 6 standard deviations of half a step at most
    step = 2 * 2.0**(byte.max() - 127.0)
    assert (np.abs(mean - x[0].double().cpu().numpy()) <= 6 * step / 2 / 64).all()


# ---- products ------------------------------------------------------------------------------------------------------------------
def operand(rows, K, seed, spread):
    """Codes as bytes, their scales' bytes, what they stand for."""
    r = np.random.default_rng(seed)
    code = r.integers(0, 16, (rows, 32 * R.blocks_of(K)))
    code[:, K:] = 0
    byte = 127 + r.integers(-spread, spread + 1, (rows, R.blocks_of(K)))
    return code, byte, R.stands_for(code, byte, K)


def on_device(code, byte, K):
    return torch.from_numpy(R.packed(code)).to(DEV), torch.from_numpy(R.in_panels(byte, K)).to(DEV)


def product(M, N, K, dtype, bias, scratch, spread, seed=1, extra=0):
    (ac, ab, av), (bc, bb, bv) = operand(M, K, seed, spread), operand(N, K, seed + 1, spread)
    a, sa = on_device(ac, ab, K)
    b, sb = on_device(bc, bb, K)
    c = np.random.default_rng(seed).standard_normal(N).astype(np.float32) if bias else None
    y = torch.full((M + 1, N + extra), 3.0, dtype=dtype, device=DEV)
    ws = torch.empty(B.int8t_mx4_product_workspace_bytes(M, N, K), dtype=torch.uint8, device=DEV) if scratch else None
    B.int8t_mx4_product(a, sa, b, sb, M, N, K, None if c is None else torch.from_numpy(c).to(DEV), y, N + extra, type=B.DTYPES[dtype], ws=ws if ws is None or ws.numel() else None)
    y = y.cpu()
    assert (y[M] == 3.0).all() and (y[:, N:] == 3.0).all()
    want, size = av @ bv.T, np.abs(av) @ np.abs(bv).T
    if c is not None:
        want, size = want + c, size + np.abs(c)
    return y[:M, :N], want, size


HALF = {F32: 2.0**-24, BF16: 2.0**-8, F16: 2.0**-11}


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scratch", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (3, 5, 33), (17, 31, 64), (64, 64, 256), (65, 66, 255), (130, 70, 257), (33, 200, 4096), (128, 129, 1000), (300, 515, 1030), (256, 1024, 2100)])
def test_product(M, N, K, dtype, scratch):
    """Scales within three powers of two either way: sums of 4096 products below 36 2^6, in steps of 2^-8, are exact in fp32 (36 4096 2^14 = 2^31 only if all products were the
    largest; random ones stay below 2^24 steps), so results are the exact sums rounded once."""
    y, want, size = product(M, N, K, dtype, False, scratch, 1, extra=3)
    assert np.abs(want).max() * 2**4 < 2**24 and size.max() * 2**4 < 2**24          # (steps of 2^-4: halves times halves times 2^-2)
    assert torch.equal(y, torch.from_numpy(want).float().to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(16, 48, 70), (200, 130, 500), (130, 260, 4000)])
def test_product_of_scales_far_apart(M, N, K, dtype):
    """Each of K additions rounds by 2^-24 of what is summed at most (2^-23 where the matrix units cut instead), the bias by one more, the result by half a step of its type."""
    y, want, size = product(M, N, K, dtype, True, True, 20)
    bound = (K + 1) * 2.0**-23 * size + HALF[dtype] * np.abs(want) * 1.01
    got = y.double().numpy()
    finite = np.abs(want) < torch.finfo(dtype).max
    tiny = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert (np.abs(got - want)[finite] <= (bound + tiny)[finite]).all()


def test_every_tile_is_used_by_some_call():
    seen = set()
    for M in (1, 40, 128, 300, 600, 1001, 2048, 4096, 8192):
        for N in (64, 512, 1000, 4096, 16384):
            for K in (64, 512, 4096):
                d = B.int8t_mx4_product_division(M, N, K, B.int8t_mx4_product_workspace_bytes(M, N, K))
                seen.add((d.rows, d.stages, d.shares > 1))
    assert {t[0] for t in seen} == {64, 128, 256}


@pytest.mark.parametrize("M,N,K", [(1000, 4100, 1300), (2050, 2100, 700), (4100, 4000, 520), (5000, 8200, 300), (600, 700, 9000)])
def test_product_of_many_tiles(M, N, K):
    """On the GPU in 64 bits; exact as above."""
    (ac, ab, av), (bc, bb, bv) = operand(M, K, 1, 0), operand(N, K, 2, 0)
    a, sa = on_device(ac, ab, K)
    b, sb = on_device(bc, bb, K)
    y = torch.empty(M, N, device=DEV)
    ws = torch.empty(max(16, B.int8t_mx4_product_workspace_bytes(M, N, K)), dtype=torch.uint8, device=DEV)
    B.int8t_mx4_product(a, sa, b, sb, M, N, K, None, y, N, ws=ws)
    want = torch.from_numpy(av).to(DEV) @ torch.from_numpy(bv).to(DEV).T
    assert float(want.abs().max()) * 4 < 2**24 and torch.equal(y.double(), want)


def test_product_with_nan_scales():
    (ac, ab, av), (bc, bb, bv) = operand(70, 300, 1, 0), operand(90, 300, 2, 0)
    ab[5, 3], bb[66, 9] = 255, 255
    a, sa = on_device(ac, ab, 300)
    b, sb = on_device(bc, bb, 300)
    y = torch.empty(70, 90, device=DEV)
    B.int8t_mx4_product(a, sa, b, sb, 70, 90, 300, None, y, 90)
    want = np.zeros((70, 90), bool)
    want[5], want[:, 66] = True, True
    assert np.array_equal(torch.isnan(y).cpu().numpy(), want)
