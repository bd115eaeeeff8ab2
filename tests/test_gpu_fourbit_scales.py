"""Attention over 4-bit caches whose scales are at the ends of their range: finite values of any size have a finite mean, and none are lost.  The reference is in 64 bits; bounds are
those of check_attend()."""
import math
import os
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

from test_gpu_fourbit_cache import attend_reference, check_attend, division, make_cache, queries, starts_of  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16


def rescale(scales, low, high, seed, blocks=False):
    """Bytes from low to high in place of those of keys in use, the same for all blocks of a key's row, or one for each block."""
    g = torch.Generator().manual_seed(seed)
    new = torch.randint(low, high + 1, scales.shape if blocks else scales.shape[:-1] + (1,), generator=g).to(torch.uint8).expand(scales.shape).to(DEV)
    scales.copy_(torch.where(scales == 255, scales, new))


def check(cache, q, starts, lengths, table, rows, floor):
    """check_attend()'s bound with another floor, which may go by the largest score."""
    dtype, width = q.dtype, max(len(t) for t in table)
    assert division(cache, q, len(lengths), width, True).rows == rows
    want, absolute, _, size = attend_reference(cache, q, starts, lengths, table, True, cache.dim ** -0.5)
    t = torch.zeros(len(table), width, dtype=torch.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    got = cache.attend(q, *(torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, lengths)), t.to(DEV)).cpu().double()
    e_p = {F32: 2.0**-23, BF16: 2.0**-16}[dtype] if rows == 16 else {F32: 2.0**-20, BF16: 2.0**-11}[dtype]
    ds, e_sum = 2.0**-17 * size + 2.0**-20, (max(lengths) / 32 + 40) * 2.0**-23
    bound = (2 * ds[..., None] + e_p + e_sum) * absolute + {F32: 2.0**-24, BF16: 2.0**-8}[dtype] * 1.01 * want.abs() + (floor(float(size.max())) if callable(floor) else floor)
    assert bool(((got - want).abs() <= bound).all()), ((got - want).abs() / bound).max()
    return got


def floor_of_p(cache, lengths):
    """p is held down to 2^-126 of the row's unit, and the unit is at most the largest score plus 29 + log2(keys) - 5 for the largest values, less what these fall short of 2^125:
    each of the keys may be off by as much of the largest value, in sums of p of at least 2^-(that)."""
    most, keys = int(cache.vs[cache.vs < 253].max()), max(lengths)
    return keys * 2.0 ** (-126 + max(0, most - 229 + max(0.0, math.log2(keys) - 5))) * 6 * 2.0 ** (most - 127)


# (heads, group, dim, page, new tokens, lengths): single tokens in blocks of eight waves and of four, ragged chunks, shares that are joined
ROWS = [(2, 4, 128, 16, [1] * 5, [1, 40, 129, 16, 33]), (1, 5, 64, 24, [1, 1], [700, 90]), (1, 2, 80, 7, [3, 20], [50, 33]), (1, 3, 256, 16, [2, 9], [61, 40]), (1, 5, 64, 16, [1, 1], [5000, 2049]),
        (16, 4, 64, 16, [1] * 40, [20 + 7 * b for b in range(40)])]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low,high,blocks", [(252, 252, False), (236, 242, False), (226, 252, True), (198, 206, True)])
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", ROWS)
def test_large_values(dtype, low, high, blocks, heads, group, dim, page, new, lengths):
    """Bytes up to 252: values of 6 2^125.  Scores differ by tens, so that p grows over those of the first keys."""
    cache, table = make_cache(lengths, heads, dim, page)
    rescale(cache.vs, low, high, 3, blocks)
    got = check(cache, queries(sum(new), heads * group, dim, dtype, size=8.0), starts_of(new), lengths, table, 16, floor_of_p(cache, lengths))
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_values_of_keys_that_are_hardly_seen(dtype):
    """A key whose score is 85 (2^122) below the others', but whose values are 2^123 times theirs, counts; one that is not seen does not take the others' bits."""
    heads, dim, n = 1, 64, 96
    cache, table = make_cache([n, n], heads, dim, 16)
    cache.kq.zero_(), cache.ks.copy_(torch.where(cache.ks == 255, cache.ks, torch.full_like(cache.ks, 127)))
    rescale(cache.vs, 127, 127, 0)
    page = table[0][3]                           # (keys 48 to 63 of the first request)
    cache.kq[page, 0, 5, 0] = 0x0F               # -6 in the first dim
    cache.vs[page, 0, 5] = 250
    page = table[1][5]
    cache.kq[page, 0, 15, 0] = 0x07              # the second request's last key: +6, large values, and behind what its first token sees
    cache.vs[page, 0, 15] = 252
    q = torch.zeros(4, 2, dim, dtype=dtype, device=DEV)
    q[:2, :, 0] = 113.0                          # 6 113 / 8 = 84.75
    q[2:, :, 0] = 1.0
    got = check_attend(cache, q, [0, 2, 4], [n, n], table, rows=16)
    assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low,high", [(1, 14), (1, 40), (30, 60)])
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", ROWS)
def test_small_keys(dtype, low, high, heads, group, dim, page, new, lengths):
    """Queries make up for them."""
    cache, table = make_cache(lengths, heads, dim, page)
    rescale(cache.ks, low, high, 3)
    check_attend(cache, queries(sum(new), heads * group, dim, dtype) * 2.0 ** (125 - high), starts_of(new), lengths, table, rows=16)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("low,high", [(1, 14), (13, 30), (30, 60)])
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", ROWS)
def test_small_values(dtype, low, high, heads, group, dim, page, new, lengths):
    """Products and sums below the least normal fp32 number, 2^-126, may be zeros, one for each key."""
    cache, table = make_cache(lengths, heads, dim, page)
    rescale(cache.vs, low, high, 3)
    check(cache, queries(sum(new), heads * group, dim, dtype), starts_of(new), lengths, table, 16, max(lengths) * 2.0**-125)


# Larger blocks: 128 rows, 256, and keys in shares
LARGER = [(16, 8, 64, 16, [170, 0, 129, 3], [300, 9, 140, 64], 128), (40, 4, 128, 16, [300, 77, 1, 130], [500, 77, 40, 131], 256), (4, 8, 64, 24, [256], [8200], 128)]


@pytest.mark.parametrize("heads,group,dim,page,new,lengths,rows,dtype", [c + (t,) for c in LARGER for t in (F32, BF16) if t is BF16 or c[2] == 64])
@pytest.mark.parametrize("low,high,blocks", [(252, 252, False), (232, 252, True)])
def test_large_values_in_larger_blocks(dtype, low, high, blocks, heads, group, dim, page, new, lengths, rows):
    """A row's largest weight, p times its row's factor of 2^(byte - 140) at most, is 2^14 at least, so that l is at least 2^(154 - byte); p below 2^-126 is zero, off by as much of a value for
    each of the keys.  Steps of the weights as in check_attend()."""
    cache, table = make_cache(lengths, heads, dim, page)
    rescale(cache.vs, low, high, 3, blocks)
    most, value = int(cache.vs[cache.vs < 253].max()), 6 * 2.0 ** (high - 127)
    floor = max(lengths) * value * (2.0**-38 + 2.0 ** (-126 - (154 - most)))
    assert torch.isfinite(check(cache, queries(sum(new), heads * group, dim, dtype), starts_of(new), lengths, table, rows, floor)).all()


@pytest.mark.parametrize("heads,group,dim,page,new,lengths,rows", [c for c in LARGER if c[2] == 64])
@pytest.mark.parametrize("low,high", [(1, 13), (1, 40)])
def test_small_keys_in_larger_blocks(low, high, heads, group, dim, page, new, lengths, rows):
    cache, table = make_cache(lengths, heads, dim, page)
    rescale(cache.ks, low, high, 3)
    check_attend(cache, queries(sum(new), heads * group, dim, F32) * 2.0 ** (125 - high), starts_of(new), lengths, table, rows=rows)


@pytest.mark.parametrize("heads,group,dim,page,new,lengths,rows,dtype", [c + (t,) for c in LARGER for t in (F32, BF16) if t is BF16 or c[2] == 64])
@pytest.mark.parametrize("low,high,blocks", [(1, 13, False), (0, 16, True), (13, 30, False)])
def test_small_values_in_larger_blocks(dtype, low, high, blocks, heads, group, dim, page, new, lengths, rows):
    """Positive values, and scores near each other.  p reaches 2^109 at least, so that l is at least n 2^109 e^(-2 largest score); weights p vs are rounded to steps of 2^-24, by 2^-25 at most
    each, and multiply codes of 6 2^13 at most:  n 2^-25 6 2^13 / l.  Results below the least normal number as in check()."""
    cache, table = make_cache(lengths, heads, dim, page)
    rescale(cache.vs, low, high, 3, blocks)
    cache.vq.bitwise_and_(0x77)
    q = queries(sum(new), heads * group, dim, dtype, size=0.02)
    check(cache, q, starts_of(new), lengths, table, rows, lambda score: 2.0**-25 * 6 * 2.0**13 * 2.0**-109 * math.exp(2 * score) + 2.0**-125)
