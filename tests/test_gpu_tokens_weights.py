"""Attention's weights (softmax times the values' scales) row by row: keys that a row does not see, value scales far apart, sums of any size."""
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

from paper_1912_12607_amd import tokens  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
E_P = {F32: 2.0**-20, BF16: 2.0**-10.9, F16: 2.0**-10.9}        # p times a value scale: 22 bits or 11, exponentials
E_OUT = {F32: 2.0**-22, BF16: 2.0**-8, F16: 2.0**-10.9}         # the result's rounding


def cache_of(lengths, heads, dim, page, seed, spread=0.5):
    """A cache that those requests fill, pages in random order, and their tables."""
    gen = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    pages = sum(need) + 1
    ids = torch.randperm(pages, generator=gen).tolist()
    table = torch.zeros(len(lengths), max(1, max(need)), dtype=torch.int32)
    for b, n in enumerate(need):
        table[b, :n] = torch.tensor([ids.pop() for _ in range(n)], dtype=torch.int32)
    q = [torch.randint(-127, 128, (pages, heads, page, dim), generator=gen, dtype=torch.int8).to(DEV) for _ in range(2)]
    s = [(torch.exp(spread * torch.randn(pages, heads, page, generator=gen)) / 64).to(DEV) for _ in range(2)]
    return tokens.PagedCache(q[0], s[0], q[1], s[1]), table.to(DEV)


def places(table, b, keys, page):
    """Indices (page, row) of those keys of request b."""
    keys = torch.as_tensor(keys, device=DEV)
    return table[b].long()[keys // page], keys % page


def queries(T, heads, dim, dtype, seed, size=1.5):
    return (torch.randn(T, heads, dim, generator=torch.Generator().manual_seed(seed)) * size).to(dtype).to(DEV)


def ints(*lists):
    return [torch.tensor(v, dtype=torch.int32, device=DEV) for v in lists]


def starts_of(new):
    out = [0]
    for n in new:
        out.append(out[-1] + n)
    return out


def in_64_bits(cache, q, starts, lengths, table, causal=True):
    """(output, sum p |v| / sum p, largest p vs / sum p, logarithm of sum p, largest sum of |terms| of a score) of every row."""
    T, HQ, D = q.shape
    H, page = cache.heads, cache.page_size
    G = HQ // H
    f64 = dict(dtype=torch.float64, device=DEV)
    out, absolute, top = torch.zeros(T, HQ, D, **f64), torch.zeros(T, HQ, D, **f64), torch.zeros(T, HQ, **f64)
    lse, size = torch.full((T, HQ), -math.inf, **f64), torch.zeros(T, HQ, **f64)
    for b, L in enumerate(lengths):
        n = starts[b + 1] - starts[b]
        if not n or not L:
            continue
        ids = table[b, :-(-L // page)].long()
        at = slice(starts[b], starts[b + 1])
        for hq in range(HQ):
            h = hq // G
            (k, _), (v, vs) = (((c[ids, h].double() * s[ids, h].double()[..., None]).reshape(-1, D)[:L], s[ids, h].double().reshape(-1)[:L])
                               for c, s in ((cache.kq, cache.ks), (cache.vq, cache.vs)))
            rows = q[at, hq].double()
            a = rows @ k.t().contiguous() / math.sqrt(D)
            if causal:
                a = a.masked_fill(torch.arange(L, device=DEV) > (L - n + torch.arange(n, device=DEV))[:, None], -math.inf)
            p = torch.exp(a - a.amax(1, keepdim=True).clamp(min=-1e300))              # (torch's softmax of doubles loses what is below 1e-38)
            p = p / p.sum(1, keepdim=True).clamp(min=1e-300)
            out[at, hq], absolute[at, hq], top[at, hq] = p @ v, p @ v.abs(), (p * vs).amax(1)
            lse[at, hq] = torch.logsumexp(a, 1)
            size[at, hq] = (rows.abs() @ k.abs().t().contiguous()).amax(1) / math.sqrt(D)
    return out, absolute, top, lse, size


def check(cache, q, starts, lengths, table, causal=True, longest=None):
    want = in_64_bits(cache, q, starts, lengths, table, causal)
    compare(cache.attend(q, *ints(starts, lengths), table, causal=causal, longest=longest, return_lse=True), want, max(lengths))


def compare(results, definition, keys):
    """Scores are off by ds (their sums in fp32, the exponential's argument), a weight p vs by e_p of itself and by 2^-39 of its row's largest (fp16 below
    2^-14 is a fixed point with steps of 2^-24, errs by half of one, and the largest weight lies at 2^14 at least), each times a code of 127 at most."""
    (got, glse), (want, absolute, top, lse, size) = results, definition
    ds = 2.0**-18 * size + 2.0**-20
    bound = (2 * ds[..., None] + E_P[got.dtype]) * absolute + E_OUT[got.dtype] * want.abs() + keys * 127 * 2.0**-39 * top[..., None] + 1e-36
    if got.dtype is F16:
        bound += 2.0**-25
    off = (got.double() - want).abs() / bound
    assert bool((off <= 1).all()), float(off.max())                         # (NaN fails)
    some = torch.isfinite(lse)
    assert torch.equal(some, torch.isfinite(glse))
    assert bool(((glse.double() - lse)[some].abs() <= 2 * ds[some] + 2.0**-20 * lse[some].abs() + 2.0**-18).all())


# blocks of 16 rows, of 128 and of 256; one and several shares of the keys
FORMS = [(1, 4, 64, 16, [20, 9], [90, 300]), (2, 2, 80, 24, [3, 17], [40, 5000]), (1, 3, 128, 7, [5, 30], [60, 31]), (1, 1, 256, 32, [12, 1], [2500, 77]),
         (1, 4, 64, 16, [200, 40], [700, 40]), (1, 4, 128, 64, [300, 150], [3000, 151]), (2, 8, 128, 16, [170], [6000]), (1, 8, 256, 32, [90, 70], [90, 1300]),
         (1, 4, 96, 24, [300], [301]), (8, 4, 64, 16, [200, 160], [700, 160]), (8, 4, 128, 64, [300, 150], [3000, 151]), (16, 8, 256, 32, [90, 70], [90, 1300]),
         (8, 4, 96, 24, [330], [331]), (4, 8, 128, 7, [150, 130], [200, 500])]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", FORMS)
@pytest.mark.parametrize("poison", [1e10, 1e30, float("inf"), float("nan")])
def test_keys_behind_a_row_do_not_reach_it(dtype, heads, group, dim, page, new, lengths, poison):
    """The causal limit hides a token's later neighbours, whose places may hold anything: rows before them are what they are without."""
    cache, table = cache_of(lengths, heads, dim, page, 1)
    starts = starts_of(new)
    q = queries(sum(new), heads * group, dim, dtype, 2)
    want = in_64_bits(cache, q, starts, lengths, table)
    before = torch.zeros(sum(new), dtype=torch.bool, device=DEV)
    for b, (n, L) in enumerate(zip(new, lengths)):
        seen = n // 2                                                       # tokens that see none of the places that are spoiled
        before[starts[b]:starts[b] + seen] = True
        p, r = places(table, b, list(range(max(0, L - n + seen), L)), page)
        for s in (cache.vs, cache.ks):
            s[p, :, r] = poison
    got = cache.attend(q, *ints(starts, lengths), table, return_lse=True)
    compare([t[before] for t in got], [t[before] for t in want], max(lengths))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", FORMS)
@pytest.mark.parametrize("causal", [True, False])
def test_value_scales_far_apart(dtype, heads, group, dim, page, new, lengths, causal):
    """Value scales over many orders of magnitude, scores that make a row attend to small ones beside the largest: a row's error is measured by its own weights.
    fp16 results: scales whose outputs its range holds."""
    cache, table = cache_of(lengths, heads, dim, page, 3)
    gen = torch.Generator().manual_seed(4)
    cache.ks.mul_(4.0)
    for b, L in enumerate(lengths):                                         # runs of tokens of like size, and single ones in between
        size = torch.linspace(-1, 1, L) + 0.3 * torch.randn(L, generator=gen)
        size = 10.0 ** ((size * 12 - 10).clamp(-24, 8) if dtype is not F16 else (size * 3 - 3).clamp(-8, 1))
        p, r = places(table, b, list(range(L)), page)
        cache.vs[p, :, r] = size.float().to(DEV)[:, None] / 64
    check(cache, queries(sum(new), heads * group, dim, dtype, 5), starts_of(new), lengths, table, causal)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim,group", [(64, 2), (128, 4), (256, 1)])
@pytest.mark.parametrize("new", [1, 400, 10000])
@pytest.mark.parametrize("scale", [0.0, 1e-30, 1e-10, 1.0, 1e20, 1e33])
def test_sums_over_many_keys(dtype, dim, group, new, scale):
    """A million keys of like weight in one share: the sum of p and its logarithm, whatever the size of the values.  The sum of weights times codes is
    formed in at most L / 16 additions in fp32, each off by 2^-24 of a sum that is no larger than the last."""
    page, L = 1024, (1 << 20) - 5
    cache = tokens.PagedCache.empty(1, page, 1, dim, DEV)
    cache.kq.fill_(100)
    cache.ks.fill_(0.5)
    cache.vq.copy_((torch.arange(dim, device=DEV) - dim // 2).clamp(-127, 127).to(torch.int8).expand(1, 1, page, dim))
    cache.vs.fill_(scale)
    q = torch.zeros(new, group, dim, dtype=dtype, device=DEV)
    table = torch.zeros(1, page, dtype=torch.int32, device=DEV)
    got, lse = cache.attend(q, *ints([0, new], [L]), table, causal=False, longest=1, return_lse=True)
    assert bool(((lse.double() - math.log(L)).abs() <= 2.0**-18).all())
    want = cache.vq[0, 0, 0].double() * cache.vs[0, 0, 0].double()
    assert bool(((got.double() - want).abs() <= (E_P[dtype] + E_OUT[dtype] + L / 16 * 2.0**-24) * want.abs()).all())


SHARED = [(2, 4, 64, 16, [1, 1], [9000, 40]), (1, 3, 256, 24, [1, 2], [40, 6000]), (1, 2, 128, 7, [20], [5000])] + FORMS


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", SHARED)
def test_nan_shows_in_rows_that_meet_it(dtype, heads, group, dim, page, new, lengths):
    """A query of NaN, a key's or a value's scale of NaN: NaN for the rows that they belong to (a value's: not in the sum's logarithm), nothing for the others."""
    starts = starts_of(new)
    T, longest = sum(new), lengths.index(max(lengths))
    for where in ("q", "k", "v"):
        cache, table = cache_of(lengths, heads, dim, page, 7)
        q = queries(T, heads * group, dim, dtype, 8)
        want = in_64_bits(cache, q, starts, lengths, table)
        hit = torch.zeros(T, heads * group, dtype=torch.bool, device=DEV)
        if where == "q":
            t = starts[longest + 1] - 1
            q[t, 0, dim - 1] = float("nan")
            hit[t, 0] = True
        else:
            n, L = new[longest], lengths[longest]
            at = L - max(1, n // 2)                                       # a key that the request's last tokens see
            p, r = places(table, longest, [at], page)
            (cache.ks if where == "k" else cache.vs)[p, heads - 1, r] = float("nan")
            hit[starts[longest + 1] - (L - at):starts[longest + 1], (heads - 1) * group:] = True
        got, lse = cache.attend(q, *ints(starts, lengths), table, return_lse=True)
        assert bool(got[hit].isnan().all()), where
        assert bool(lse[hit].isnan().all()) == (where != "v"), where
        compare([t[~hit] for t in (got, lse)], [t[~hit] for t in want], max(lengths))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,group,dim,page,new,lengths", [(8, 4, 128, 16, [1] * 12, [1500, 1, 40, 2049, 0, 700, 3, 1024, 1025, 90, 33, 5000]), (2, 1, 64, 24, [13, 2], [20, 4000]),
                                                              (1, 2, 256, 7, [1], [3]), (64, 1, 64, 16, [14] * 20, [1500] * 19 + [3])])
def test_tables_much_longer_than_the_requests(dtype, heads, group, dim, page, new, lengths):
    """The division of the keys goes by the table where `longest` is not given: most shares have none, or all keys lie in the first."""
    cache, table = cache_of(lengths, heads, dim, page, 9)
    wide = torch.full((len(new), 300000 // page), 0x7FFFFFF0, dtype=torch.int32, device=DEV)
    wide[:, :table.shape[1]] = table
    check(cache, queries(sum(new), heads * group, dim, dtype, 10), starts_of(new), lengths, wide)
