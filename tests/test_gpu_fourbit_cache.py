"""A paged cache of microscaled 4-bit codes and attention over it, against plain implementations in 64 bits on the CPU."""
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

import fourbit_reference as R  # noqa: E402
from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import fourbit  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


# ---- write, read -----------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count,heads,dim,page", [(1, 1, 16, 1), (5, 3, 48, 7), (37, 2, 64, 16), (40, 2, 80, 24), (33, 2, 128, 16), (20, 1, 144, 5), (9, 4, 256, 32)])
def test_cache_write_and_read(dtype, count, heads, dim, page):
    r = np.random.default_rng(count)
    pages = 2 * count // page + 3
    cache = fourbit.PagedCache4.empty(pages, page, heads, dim, DEV)
    for t in (cache.kq, cache.vq, cache.ks, cache.vs):
        t.fill_(0x77)
    # (tokens, heads, dim) inside of a wider tensor
    x = torch.from_numpy((r.standard_normal((count, 2 * heads + 1, dim)) * np.exp(r.standard_normal((count, 2 * heads + 1, 1)))).astype(np.float32)).to(dtype).to(DEV)
    k, v = x[:, :heads], x[:, heads:2 * heads]
    slots = torch.from_numpy(r.permutation(pages * page)[:count])
    if count > 4:
        slots[2], slots[3] = -1, pages * page                # no place
    cache.write(k, v, slots.to(DEV))
    for t, q, s in ((k, cache.kq, cache.ks), (v, cache.vq, cache.vs)):
        wq, ws = np.full(tuple(q.shape), 0x77, np.uint8), np.full(tuple(s.shape), 0x77, np.uint8)
        code, byte = R.quantise(t.double().cpu().numpy().reshape(-1, dim))
        code, byte = R.packed(code).reshape(count, heads, -1), byte.reshape(count, heads, -1)
        for i, at in enumerate(slots.tolist()):
            if 0 <= at < pages * page:
                wq[at // page, :, at % page], ws[at // page, :, at % page] = code[i], byte[i]
        assert np.array_equal(q.cpu().numpy(), wq) and np.array_equal(s.cpu().numpy(), ws)
    gk, gv = cache.read(slots.to(DEV), dtype)
    for t, got in ((k, gk), (v, gv)):
        want = R.rounded(t.double().cpu().numpy().reshape(-1, dim)).reshape(count, heads, dim)
        live = ((slots >= 0) & (slots < pages * page)).numpy()
        want[~live] = 0.0
        assert got.dtype == dtype and torch.equal(got.cpu(), torch.from_numpy(want).float().to(dtype))


def test_cache_of_no_tokens_and_nan():
    cache = fourbit.PagedCache4.empty(3, 4, 2, 64, DEV)
    none = torch.zeros(0, 2, 64, device=DEV)
    cache.write(none, none, torch.zeros(0, dtype=torch.int64, device=DEV))
    assert cache.read(torch.zeros(0, dtype=torch.int64, device=DEV))[0].shape == (0, 2, 64)
    k = torch.randn(2, 2, 64, device=DEV)
    k[1, 0, 40] = float("nan")
    k[0, 1, 3] = float("inf")
    cache.write(k, k, torch.tensor([5, 6], device=DEV))
    got, _ = cache.read(torch.tensor([5, 6], device=DEV))
    want = torch.zeros(2, 2, 64, dtype=torch.bool)
    want[1, 0, 32:], want[0, 1, :32] = True, True
    assert torch.equal(torch.isnan(got).cpu(), want)


# ---- attention -------------------------------------------------------------------------------------------------------------------
def attend_reference(cache, q, starts, lengths, table, causal, scale):
    """64 bits: (output, sum of p |v| / sum of p, logarithm of the sum, largest scale sum |q k| of a row)."""
    keys, vals = R.cache_values(cache)
    T, HQ, D = q.shape
    H, page = cache.heads, cache.page_size
    G = HQ // H
    out, absolute = torch.zeros(T, HQ, D, dtype=torch.float64), torch.zeros(T, HQ, D, dtype=torch.float64)
    lse, size = torch.full((T, HQ), -math.inf, dtype=torch.float64), torch.zeros(T, HQ, dtype=torch.float64)
    q = q.cpu().double()
    for b in range(len(lengths)):
        n, L = starts[b + 1] - starts[b], lengths[b]
        js = [j for j in range(L) if 0 <= table[b][j // page] < cache.pages]
        if not n or not js:
            continue
        p_ids, o_ids, js = torch.tensor([table[b][j // page] for j in js]), torch.tensor([j % page for j in js]), torch.tensor(js)
        t = slice(starts[b], starts[b] + n)
        end = torch.arange(L - n + 1, L + 1) if causal else torch.full((n,), L)
        seen = js[None, :] < end[:, None]
        some = seen.any(1)
        for hq in range(HQ):
            k, v = keys[p_ids, hq // G, o_ids], vals[p_ids, hq // G, o_ids]
            s = (q[t, hq] @ k.T * scale).masked_fill(~seen, -math.inf)
            top = s.max(1).values
            p = torch.where(some[:, None], torch.exp(s - top[:, None]), torch.zeros_like(s))
            total = p.sum(1).clamp(min=1e-300)[:, None]
            out[t, hq], absolute[t, hq] = p @ v / total, p @ v.abs() / total
            lse[t, hq] = torch.where(some, top + torch.log(total[:, 0]), lse[t, hq])
            size[t, hq] = (q[t, hq].abs() @ k.abs().T).masked_fill(~seen, 0.0).max(1).values * abs(scale)
    return out, absolute, lse, size


def division(cache, q, n, width, causal, longest=None):
    d = B.AttendDesc(q.shape[0], n, q.shape[1] // cache.heads, width, 0 if longest is None else longest, B.DTYPES[q.dtype], int(causal), 1.0, q.stride(0), q.stride(1), width)
    return B.int8t_mx4_cache_attend_division(cache._c, d)


def check_attend(cache, q, starts, lengths, table, causal=True, scale=None, longest=None, rows=None):
    """Bound of an element: scores carry errors of their fp32 sums (some hundred additions of 2^-24 of the sum of |terms| at most, 2^-17 of it), and of the exponential's
    argument and result, 2^-20: ds.  p is rounded to two pieces of bf16, 2^-17 of it, for fp32 to three, 2^-24; in larger blocks to one fp16, 2^-12, or two, 2^-22, with steps of
    2^-39 of the largest of p times its value's scale, and there fp32's q too.  Sums of the keys, 32 at a time, in fp32, and of the shares: (keys / 32 + 40) 2^-23.  The output to
    half a step of its type:  (2 ds + e_p + e_sum) (sum p |v| / sum p) + e_out |o| + floor."""
    dt = q.dtype
    scale_ = 1 / math.sqrt(cache.dim) if scale is None else scale
    width = max(1, max(len(t) for t in table)) if table else 1
    how = division(cache, q, len(lengths), width, causal, longest)
    if rows is not None:
        assert how.rows == rows, how.rows
    large = how.rows > 16
    e_p = {F32: 2.0**-20, BF16: 2.0**-11, F16: 2.0**-11}[dt] if large else {F32: 2.0**-23, BF16: 2.0**-16, F16: 2.0**-16}[dt]
    e_out = {F32: 2.0**-24, BF16: 2.0**-8, F16: 2.0**-11}[dt]
    want, absolute, lse, size = attend_reference(cache, q, starts, lengths, table, causal, scale_)
    t = torch.full((len(table), width), 0x7FFFFFF0, dtype=torch.int32)       # (what no length needs is not looked at)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, lengths)]
    got, glse = cache.attend(q, args[0], args[1], t.to(DEV), causal=causal, scale=scale, longest=longest, return_lse=True)
    assert got.dtype == dt and got.shape == q.shape
    # (rows behind the last request's are not written)
    last = starts[-1]
    got, glse, want, absolute, lse, size = got[:last].cpu().double(), glse[:last].cpu().double(), want[:last], absolute[:last], lse[:last], size[:last]
    ds = 2.0**-17 * size + 2.0**-20
    e_sum = (max(lengths, default=0) / 32 + 40) * 2.0**-23
    used = cache.vs[cache.vs < 253]
    floor = max(lengths, default=0) * 6 * 2.0**(float(used.max()) - 127 - 38) if large and used.numel() else 0.0
    bound = (2 * ds[..., None] + e_p + e_sum) * absolute + e_out * 1.01 * want.abs() + floor + 1e-30
    if dt is F16:
        bound = bound + 2.0**-25                                            # (smallest fp16 step, halved)
        # (what is 65520 or more, half a step above the largest, rounds to infinity)
        got = torch.where(torch.isinf(got) & (got.sign() == want.sign()) & (want.abs() + bound >= 65520.0), want, got)
    assert bool(((got - want).abs() <= bound).all()), ((got - want).abs() / bound).max()
    none = torch.isinf(lse)
    assert torch.equal(none, torch.isinf(glse) & (glse < 0)) and not got[none].any()
    assert bool(((glse - lse)[~none].abs() <= 2 * ds[~none] + e_sum + 2.0**-20 * lse[~none].abs() + 2.0**-18).all())
    return got


def make_cache(lengths, heads, dim, page, seed=0, extra=2, poison=True, spread=2):
    """A cache with the pages of requests of those lengths in random order; what no request uses holds scales of 255 and codes that are not zero."""
    r = np.random.default_rng(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + extra
    ids = r.permutation(pages).tolist()
    table = [[ids.pop() for _ in range(n)] for n in need]
    blocks = R.blocks_of(dim)
    code = r.integers(0, 16, (2, pages, heads, page, 32 * blocks))
    code[..., dim:] = 0
    q = torch.from_numpy((code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8))
    s = torch.from_numpy((125 + r.integers(-spread, spread + 1, (2, pages, heads, page, blocks))).astype(np.uint8))
    if poison:
        used = torch.zeros(pages, page, dtype=torch.bool)
        for row, n in zip(table, lengths):
            for j in range(n):
                used[row[j // page], j % page] = True
        s[~used[None, :, None].expand(2, pages, heads, page)] = 255
    return fourbit.PagedCache4(q[0].to(DEV), s[0].to(DEV), q[1].to(DEV), s[1].to(DEV), dim), table


def queries(T, heads, dim, dtype, seed=1, size=1.5):
    return (torch.randn(T, heads, dim, generator=torch.Generator().manual_seed(seed)) * size).to(dtype).to(DEV)


def starts_of(new):
    return np.concatenate([[0], np.cumsum(new)]).tolist()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,dim,page", [(2, 4, 128, 16), (1, 1, 64, 16), (3, 7, 96, 32), (2, 3, 80, 24), (1, 16, 256, 64), (2, 17, 48, 7), (4, 2, 16, 1), (1, 5, 144, 48), (2, 8, 224, 13)])
def test_attend_single_tokens(dtype, heads, group, dim, page):
    lengths = [1, 40, 0, 129, 16, 33]
    cache, table = make_cache(lengths, heads, dim, page)
    check_attend(cache, queries(len(lengths), heads * group, dim, dtype), list(range(len(lengths) + 1)), lengths, table, rows=16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim,page", [(2, 2, 128, 16), (1, 3, 64, 24), (2, 1, 256, 32), (1, 5, 80, 7)])
def test_attend_chunks(dtype, causal, heads, group, dim, page):
    new, lengths = [20, 1, 0, 45, 7], [33, 70, 12, 45, 100]
    cache, table = make_cache(lengths, heads, dim, page)
    check_attend(cache, queries(sum(new), heads * group, dim, dtype), starts_of(new), lengths, table, causal)


LARGE = [(8, 4, 128, 16, [300, 77, 1, 130], [500, 77, 40, 131]), (8, 8, 64, 16, [170, 0, 129, 3], [300, 9, 140, 64]), (8, 8, 64, 24, [170, 129], [300, 140]),
         (8, 5, 128, 7, [210, 60], [210, 333]), (8, 6, 256, 32, [190, 100], [400, 123]), (8, 6, 224, 10, [190, 100], [400, 123]), (8, 6, 96, 64, [300, 100], [310, 700]), (10, 8, 48, 1, [180], [200])]
# ... with heads enough for larger blocks, and few of those in shares
LARGER = [(40, 4, 128, 16, [300, 77, 1, 130], [500, 77, 40, 131]), (16, 8, 64, 16, [170, 0, 129, 3], [300, 9, 140, 64]), (16, 8, 64, 24, [170, 129], [300, 140]),
          (27, 5, 128, 7, [210, 60], [210, 333]), (16, 6, 96, 64, [300, 100], [310, 700]), (27, 8, 48, 1, [180], [200]), (8, 4, 128, 16, [250, 150], [4100, 2500]), (4, 8, 64, 24, [256], [8200])]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", LARGE + LARGER)
def test_attend_of_larger_blocks(dtype, causal, heads, group, dim, page, new, lengths):
    cache, table = make_cache(lengths, heads, dim, page)
    q = queries(sum(new), heads * group, dim, dtype)
    check_attend(cache, q, starts_of(new), lengths, table, causal)


def test_larger_blocks_are_used_by_those_calls():
    for heads, group, dim, page, new, lengths in LARGER:
        cache, table = make_cache(lengths, heads, dim, page)
        for dtype in (BF16, F32):
            how = division(cache, queries(sum(new), heads * group, dim, dtype), len(new), max(len(t) for t in table), True)
            assert how.rows == (16 if dim > 128 or (dim > 64 and dtype is F32) else 128 if dim <= 64 else 256)
            assert (how.shares > 1) == (max(lengths) > 1024)


@pytest.mark.parametrize("dtype,new", [(BF16, [1] * 530), (F32, [i % 3 for i in range(513)]), (BF16, [32] * 514), (BF16, [1] * 65), (F32, [i % 3 for i in range(512)]),
                                       (F16, [0] * 64 + [3] + [0] * 63 + [2, 1]), (F32, [0, 7] * 100), (BF16, [32] * 320)])
def test_attend_of_many_requests(dtype, new):
    """More of them than a wave looks at once, and than blocks look through: single tokens, some without a token or a key, and whole larger blocks."""
    lengths = [max(n, (7 * b) % 60 if b % 50 else 2100) for b, n in enumerate(new)]          # (some in shares)
    cache, table = make_cache(lengths, 1, 64, 16)
    check_attend(cache, queries(sum(new), 4, 64, dtype), starts_of(new), lengths, table, rows=128 if new[0] == 32 else 16)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[3, 2, 2], [300, 2, 200]])
def test_attend_rows_that_see_nothing(dtype, new):
    """More new tokens than keys: the first see nothing; a request whose pages are not in the cache."""
    lengths, large = [1, 0, 20], sum(new) > 100
    heads = 24 if large else 8
    cache, table = make_cache(lengths, heads, 64, 16)
    table[2] = [cache.pages, -5]
    got = check_attend(cache, queries(sum(new), 4 * heads, 64, dtype), starts_of(new), lengths, table, rows=128 if large else 16)
    assert not got[sum(new[:1]):].any()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [16, 24])
def test_attend_long_context(dtype, page):
    """Shares of the keys, joined; a table much longer than the requests."""
    lengths = [5000, 3, 1100, 2049]
    cache, table = make_cache(lengths, 1, 64, page)
    for longest in (None, 5000):
        check_attend(cache, queries(4, 5, 64, dtype), [0, 1, 2, 3, 4], lengths, [t + [0] * (700 - len(t)) for t in table], longest=longest)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("new", [[2, 3], [300, 200]])
@pytest.mark.parametrize("spread", [12, 20])
def test_attend_scales_far_apart(dtype, new, spread):
    """Blocks of a key and of a value 2^24 and 2^40 apart, scores of hundreds: what a row sees most of is what counts.  (Blocks of larger tiles lose bits 2^36 below their row's
    largest: 2^-36 6 of it is below the bound's 2^-17.)"""
    lengths, large = [200, 333], sum(new) > 100
    heads = 24 if large else 8
    cache, table = make_cache(lengths, heads, 128, 16, spread=spread)
    check_attend(cache, queries(sum(new), 4 * heads, 128, dtype, size=2.0**-spread), starts_of(new), lengths, table, causal=False, rows=256 if large and dtype is not F32 else 16)


def test_attend_without_keys_or_pages():
    """Fewer tokens than requests, tables without a column, lengths of zero."""
    cache, _ = make_cache([20], 2, 64, 16)
    for width in (0, 3):
        for new in ([1, 0, 1], [0] * 63 + [2], [40, 0, 1]):
            q = queries(sum(new), 8, 64, BF16)
            args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts_of(new), [0] * len(new))]
            out, lse = cache.attend(q, *args, torch.zeros(len(new), width, dtype=torch.int32, device=DEV), return_lse=True)
            assert not out.any() and (lse == -math.inf).all()


def test_attend_scale_of_any_sign():
    lengths = [70, 333]
    cache, table = make_cache(lengths, 24, 64, 16)
    for new in ([1, 4], [200, 190]):
        q = queries(sum(new), 96, 64, BF16)
        for scale in (-0.3, 0.0, 2.0):
            check_attend(cache, q, starts_of(new), lengths, table, scale=scale, causal=False, rows=128 if new[0] > 1 else 16)


@pytest.mark.parametrize("new", [[1, 2], [300, 200]])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nan_reaches_the_rows_that_see_it_and_no_others(new, dtype):
    lengths, heads = [320, 260], 24
    cache, table = make_cache(lengths, heads, 64, 16)
    q = queries(sum(new), 4 * heads, 64, dtype)
    assert division(cache, q, 2, 20, True).rows == (128 if sum(new) > 100 else 16)
    starts = starts_of(new)
    args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in (starts, lengths)]
    t = torch.zeros(2, 20, dtype=torch.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    t = t.to(DEV)
    clean = cache.attend(q, *args, t)
    assert torch.isfinite(clean).all()
    for tensor, head, j, block in ((cache.ks, 3, lengths[0] - 1, 1), (cache.vs, 5, lengths[0] - 1, 0), (cache.vs, 0, 100, 1)):
        at = (table[0][j // 16], head, j % 16, block)
        before = tensor[at].clone()
        tensor[at] = 255
        got = cache.attend(q, *args, t)
        tensor[at] = before
        rows = torch.arange(sum(new), device=DEV)
        sees = (rows < new[0]) & (rows + lengths[0] - new[0] >= j)
        bad = torch.zeros(sum(new), 4 * heads, dtype=torch.bool, device=DEV)
        bad[sees, 4 * head:4 * head + 4] = True
        assert torch.equal(torch.isnan(got).all(-1), bad) and torch.equal(torch.isnan(got).any(-1), bad)
        assert torch.equal(got[~bad], clean[~bad])
    q2 = q.clone()
    q2[0, 7, 20] = float("nan")
    got = cache.attend(q2, *args, t)
    bad = torch.zeros(sum(new), 4 * heads, dtype=torch.bool, device=DEV)
    bad[0, 7] = True
    assert torch.equal(torch.isnan(got).all(-1), bad) and torch.equal(torch.isnan(got).any(-1), bad)


def test_attend_strided_queries_repeats_and_rows_behind_the_last():
    lengths = [90, 33]
    cache, table = make_cache(lengths, 2, 64, 16)
    wide = queries(9, 11, 64, BF16)
    q = wide[:, 2:10]
    a = check_attend(cache, q, [0, 4, 7], lengths, table)
    args = [torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 4, 7], lengths)]
    t = torch.zeros(2, 8, dtype=torch.int32)
    for b, row in enumerate(table):
        t[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    for tt in (t.to(DEV), torch.cat([t, t], 1).to(DEV)[:, :8], t.t().contiguous().t().to(DEV)):
        got = cache.attend(q, *args, tt)
        assert torch.equal(got[:7].cpu().double(), a)
    assert torch.equal(cache.attend(q.contiguous(), *args, t.to(DEV))[:7], got[:7])
    out, lse = torch.full((9, 8, 64), 7.0, dtype=BF16, device=DEV), torch.full((9, 8), 7.0, device=DEV)
    d = B.AttendDesc(9, 2, 4, 8, 0, B.BF16, 1, 0.125, q.stride(0), q.stride(1), 8)
    B.int8t_mx4_cache_attend(cache._c, d, q.data_ptr(), *args, t.to(DEV), out, lse)
    assert torch.equal(out[:7], got[:7]) and (out[7:] == 7.0).all() and (lse[7:] == 7.0).all()


def test_cache_beyond_four_gib():
    """Codes behind 2^32 bytes, places found in 64 bits."""
    page, heads, dim = 64, 16, 256
    pages = (9 << 29) // (page * heads * dim // 2)
    cache = fourbit.PagedCache4.empty(pages, page, heads, dim, DEV)
    assert cache.kq.numel() > 1 << 32
    k, v = (torch.randn(130, heads, dim, device=DEV) for _ in range(2))
    ids = [pages - 1, 0, pages - 2]
    slots = torch.tensor([ids[j // page] * page + j % page for j in range(130)], device=DEV)
    cache.write(k, v, slots)
    rk, rv = cache.read(slots)
    assert np.array_equal(rk.cpu().numpy().astype(np.float64), R.rounded(k.double().cpu().numpy().reshape(-1, dim)).reshape(130, heads, dim))
    small = fourbit.PagedCache4.empty(3, page, heads, dim, DEV)
    small.write(k, v, torch.arange(130, device=DEV))
    for n in (1, 130):
        q = queries(n, heads * 2, dim, BF16)
        args = [torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, n], [130])]
        assert torch.equal(cache.attend(q, *args, torch.tensor([ids], dtype=torch.int32, device=DEV)), small.attend(q, *args, torch.tensor([[0, 1, 2]], dtype=torch.int32, device=DEV)))


def test_refusals():
    cache = fourbit.PagedCache4.empty(2, 16, 2, 64, DEV)
    i32 = dict(dtype=torch.int32, device=DEV)
    s, n, t = torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros(1, 2, **i32)
    q = torch.zeros(1, 4, 64, device=DEV)
    k = torch.zeros(3, 2, 64, device=DEV)
    slots = torch.zeros(3, dtype=torch.int64, device=DEV)
    for call in (lambda: cache.write(k, k, slots[:2]), lambda: cache.write(k, k[:2], slots), lambda: cache.write(k.bfloat16(), k, slots), lambda: cache.write(k, k, slots.int()),
                 lambda: cache.read(slots.cpu()), lambda: cache.attend(q[..., :32], s, n, t), lambda: cache.attend(torch.zeros(1, 3, 64, device=DEV), s, n, t),
                 lambda: cache.attend(q, s.long(), n, t), lambda: cache.attend(q, s[:1], n, t), lambda: cache.attend(q, s, n, t[0]), lambda: cache.attend(q.cpu(), s, n, t),
                 lambda: fourbit.PagedCache4.empty(2, 16, 2, 60, DEV), lambda: fourbit.PagedCache4.empty(2, 16, 2, 272, DEV),
                 lambda: fourbit.PagedCache4(cache.kq, cache.ks, cache.vq, cache.vs, 96), lambda: fourbit.PagedCache4(cache.kq.char(), cache.ks, cache.vq, cache.vs, 64),
                 lambda: fourbit.PagedCache4(cache.kq, cache.ks[:, :, :, :1], cache.vq, cache.vs, 64)):
        with pytest.raises(RuntimeError):
            call()
    for call in (lambda: cache.read(slots, torch.float64), lambda: cache.write(k.double(), k.double(), slots)):
        with pytest.raises(TypeError):
            call()
