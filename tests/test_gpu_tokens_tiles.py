"""Every division of the work that the token operators choose by size: tiles of products with their stages and shares, blocks of attention with their waves
and shares.  The sizes are ragged, and each case asserts that its division is the one that it stands for."""
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
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import tokens  # noqa: E402
from test_gpu_tokens import codes, pad16, values  # noqa: E402
from test_gpu_tokens_weights import cache_of, check, queries, starts_of  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]


def exact_product(a, sa, b, sb, bias, dtype):
    """(float)sum * (sa * sb) + bias, each operation rounded once, in the type: sums of codes are whole in 64 bits (and below 2^31)."""
    acc = a.double() @ b.double().t().contiguous()
    y = acc.float() * (sa[:, None] * (1.0 if sb is None else sb[None]))
    return (y if bias is None else y + bias).to(dtype)


# rows of a tile, stages, divided: reductions that end at each of the stages, one shorter than the stages among them
PRODUCTS = [(64, 4, False, 1, 390, 33), (64, 4, False, 1, 17, 35), (64, 4, False, 70, 130, 34), (64, 4, False, 130, 300, 97), (64, 4, True, 1, 8200, 35),
            (64, 4, True, 3, 2049, 33), (64, 4, True, 67, 4112, 34), (64, 4, True, 1, 65000, 33), (128, 2, False, 517, 130, 7657), (128, 2, False, 467, 17, 8254),
            (128, 2, True, 4219, 33000, 65), (128, 2, True, 2095, 65000, 70), (128, 3, False, 5539, 1500, 522), (128, 3, False, 196, 3100, 14051),
            (128, 3, False, 222, 1290, 12607), (128, 3, True, 1866, 50000, 67), (128, 3, True, 70, 20011, 3170), (128, 3, True, 67, 65536, 1595),
            (256, 2, False, 1375, 390, 6138), (256, 2, False, 514, 520, 15624), (256, 2, True, 2173, 50000, 213), (256, 2, True, 157, 65000, 2695)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,stages,divided,M,K,N", PRODUCTS)
def test_products_by_every_tile(dtype, rows, stages, divided, M, K, N):
    need = B.int8t_product_workspace_bytes(M, N, K) if divided else 0
    d = B.int8t_product_division(M, N, K, need)
    assert (d.rows, d.stages, d.shares > 1) == (rows, stages, divided)
    gen = torch.Generator(device=DEV).manual_seed(M + N)

    def up(n):
        t = torch.zeros(n, pad16(K), dtype=torch.int8, device=DEV)
        t[:, :K] = torch.randint(-127, 128, (n, K), generator=gen, device=DEV, dtype=torch.int8)
        return t
    a, b = up(M), up(N)
    a[M - 1, :K], b[N - 1, :K] = 127, -127          # the largest sum there is
    sa, sb = (torch.exp(torch.randn(n, generator=gen, device=DEV)) for n in (M, N))
    bias = None if dtype is BF16 else torch.randn(N, generator=gen, device=DEV)
    pitch = N + (8 - N % 8) % 8 if dtype is BF16 else N + 1                # whole lines, and rows off 16 bytes
    y = torch.full((M, pitch), 7.0, dtype=dtype, device=DEV)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    B.int8t_product(a, sa, b, sb, M, N, K, bias, y, pitch, type=B.DTYPES[dtype], ws=ws)
    assert torch.equal(y[:, :N], exact_product(a[:, :K], sa, b[:, :K], sb, bias, dtype)) and bool((y[:, N:] == 7.0).all())


# both gradients' products in one launch, for each tile that they may share
@pytest.mark.parametrize("rows,stages,M,K,N", [(256, 2, 1530, 6133, 1501), (128, 3, 1301, 2311, 1400), (64, 4, 250, 1030, 300)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_large_layers(dtype, rows, stages, M, K, N):
    for m, k, n in ((M, N, K), (N, M, K)):
        d = B.int8t_product_division(m, n, k, B.int8t_product_workspace_bytes(m, n, k))
        assert (d.rows, d.stages, d.shares) == (rows, stages, 1)
    (x, x32), (w, w32), (g, g32) = values((M, K), 1, dtype), values((N, K), 2, dtype, 0.3), values((M, N), 3, dtype)
    x, w, seed = x.to(DEV).requires_grad_(True), w.to(DEV).requires_grad_(True), 99
    B.int8t_profile_start(None)
    y = tokens.linear(x, w, seed=seed)
    dx, dw = torch.autograd.grad(y, [x, w], g.to(DEV))
    assert B.int8t_profile_stop()["product_kernel"][0] == 2
    (xq, sx), (wq, sw) = codes(x32, 1), codes(w32, 1)
    gq, sg = codes(g32 * sw.T, 1, seed)
    hq, sh = codes(g32 * sx, 0, seed ^ (1 << 63))

    def dev(q):
        return torch.from_numpy(np.ascontiguousarray(q).astype(np.int8)).to(DEV)

    def vec(s):
        return torch.from_numpy(s.reshape(-1)).to(DEV)
    assert torch.equal(y, exact_product(dev(xq), vec(sx), dev(wq), vec(sw), None, dtype))
    assert torch.equal(dx, exact_product(dev(gq), vec(sg), dev(wq.T), None, None, dtype))
    assert torch.equal(dw, exact_product(dev(hq.T), vec(sh), dev(xq.T), None, None, dtype))


def division(cache, T, requests, group, width, dtype, longest):
    desc = B.AttendDesc(T, requests, group, width, longest, B.DTYPES[dtype], 1, 0.125, heads_of(cache, group), cache.dim, width)
    return B.int8t_cache_attend_division(cache._c, desc)


def heads_of(cache, group):
    return cache.heads * group * cache.dim


# blocks of 16 rows by four and by eight waves, with the keys whole and in shares; larger blocks whole and in shares
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
@pytest.mark.parametrize("page", [16, 24, 7])
@pytest.mark.parametrize("rows,waves,divided,heads,group,new,lengths", [
    (16, 4, False, 8, 2, [1] * 40, [1 + 23 * i for i in range(40)]), (16, 4, True, 8, 1, [1] * 20, [3000 - 150 * i for i in range(20)]),
    (16, 8, False, 2, 4, [1, 3, 2], [900, 17, 64]), (16, 8, True, 1, 4, [1, 4], [4000, 70])])
def test_attention_by_16_rows(dtype, dim, page, rows, waves, divided, heads, group, new, lengths):
    cache, table = cache_of(lengths, heads, dim, page, 1)
    d = division(cache, sum(new), len(new), group, table.shape[1], dtype, max(lengths))
    assert (d.rows, d.waves, d.shares > 1) == (rows, waves, divided)
    check(cache, queries(sum(new), heads * group, dim, dtype, 2), starts_of(new), lengths, table, longest=max(lengths))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("page", [16, 24, 7])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("divided,group,new,lengths", [(False, 4, [300, 290], [301, 500]), (True, 4, [330, 320], [3000, 2500])])
def test_attention_by_many_rows(dtype, dim, page, causal, divided, group, new, lengths):
    heads = 8
    cache, table = cache_of(lengths, heads, dim, page, 3)
    longest = max(lengths) if divided else 1
    d = division(cache, sum(new), len(new), group, table.shape[1], dtype, longest)
    want = 256 if dim == 128 and dtype is not F32 else 128
    assert (d.rows, d.waves, d.shares > 1) == (want, want // 32, divided)
    check(cache, queries(sum(new), heads * group, dim, dtype, 4), starts_of(new), lengths, table, causal, longest=longest)
