"""The binding's calls of the token operators, as a program makes that brings its own memory: the same as through the modules."""
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

from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import tokens  # noqa: E402

DEV = torch.device("cuda:0")


def normal(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("M,K,N", [(40, 70, 33), (300, 128, 200)])
def test_linear(M, K, N):
    x, w, b, g = (normal(*s, seed=i) for i, s in enumerate(((M, K), (N, K), (N,), (M, N))))
    xs, ws, bs = (t.clone().requires_grad_(True) for t in (x, w, b))
    y = tokens.linear(xs, ws, bs, seed=11)
    dx, dw, db = torch.autograd.grad(y, [xs, ws, bs], g)
    desc = B.LinearDesc(M, K, N, B.F32, B.F32)
    Kp = (K + 15) & ~15
    xq, wq = (torch.empty(n, Kp, dtype=torch.int8, device=DEV) for n in (M, N))
    sx, sw, my, mdx, mdw, mdb = (torch.full(s, 7.0, device=DEV) for s in ((M,), (N,), (M, N), (M, K), (N, K), (N,)))
    need = max(B.int8t_linear_workspace_bytes(desc, i) for i in (0, 1))
    ws_ = torch.empty(need, dtype=torch.uint8, device=DEV)
    p = B.LinearBuffers(x=x.data_ptr(), w=w.data_ptr(), dy=g.data_ptr(), x_pitch=K, w_pitch=K, y_pitch=N, dy_pitch=N, xq=xq.data_ptr(), wq=wq.data_ptr(), sx=sx.data_ptr(),
                        sw=sw.data_ptr(), bias=b.data_ptr(), y=my.data_ptr(), dx=mdx.data_ptr(), dw=mdw.data_ptr(), db=mdb.data_ptr(), ws=ws_.data_ptr(), ws_bytes=need)
    B.int8t_linear_fwd(desc, p)
    B.int8t_linear_bwd(desc, p, seed=11)
    for mine, want in ((my, y.detach()), (mdx, dx), (mdw, dw), (mdb, db)):
        assert torch.equal(mine, want)


def test_cache_and_attention():
    heads, dim, group, page, T = 2, 64, 3, 16, 50
    cache, other = (tokens.PagedCache.empty(5, page, heads, dim, DEV) for _ in range(2))
    k, v, q = normal(T, heads, dim, seed=1), normal(T, heads, dim, seed=2), normal(T, heads * group, dim, seed=3)
    slots = torch.randperm(80, generator=torch.Generator().manual_seed(4))[:T].to(DEV)
    table = torch.tensor([[3, 0, 4, 1]], dtype=torch.int32, device=DEV)
    starts, lengths = torch.tensor([0, T], dtype=torch.int32, device=DEV), torch.tensor([T], dtype=torch.int32, device=DEV)
    cache.write(k, v, slots)
    c = B.Cache(other.kq.data_ptr(), other.vq.data_ptr(), other.ks.data_ptr(), other.vs.data_ptr(), 5, page, heads, dim)
    row = heads * dim
    B.int8t_cache_write(c, k, v, B.F32, T, row, dim, row, dim, slots)
    assert all(torch.equal(getattr(cache, n), getattr(other, n)) for n in ("kq", "ks", "vq", "vs"))
    back = torch.empty_like(k), torch.empty_like(v)
    B.int8t_cache_read(c, slots, T, *back, B.F32)
    assert all(torch.equal(a, b) for a, b in zip(back, cache.read(slots)))
    want, lse = cache.attend(q, starts, lengths, table, return_lse=True)
    d = B.AttendDesc(T, 1, group, 4, 0, B.F32, 1, dim ** -0.5, heads * group * dim, dim, 4)
    need = B.int8t_cache_attend_workspace_bytes(c, d)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV) if need else None
    out, mine = torch.empty_like(q), torch.empty(T, heads * group, device=DEV)
    B.int8t_cache_attend(c, d, q, starts, lengths, table, out, mine, ws)
    assert torch.equal(out, want) and torch.equal(mine, lse)
