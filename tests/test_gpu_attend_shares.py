"""Attention whose keys are dealt out in shares that a second pass joins: tokens that no request has are left as they were."""
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
from paper_1912_12607_amd import fourbit, tokens  # noqa: E402

DEV = torch.device("cuda:0")


@pytest.mark.parametrize("mx", [False, True])
@pytest.mark.parametrize("heads,dim,starts,T,rows", [(8, 128, [0, 4, 7], 9, 16), (8, 64, [2, 4, 7], 9, 16), (4, 128, [0, 512, 1024], 1100, 256), (4, 64, [3, 515, 1027], 1100, 128),
                                                     (8, 64, [0, 0, 0], 5, 16)])
def test_tokens_of_no_request_are_left_as_they_were(mx, heads, dim, starts, T, rows):
    group, page, pages, dtype = 4, 16, 512, torch.bfloat16
    kind, divide, attend = ((fourbit.PagedCache4, B.int8t_mx4_cache_attend_division, B.int8t_mx4_cache_attend) if mx else
                            (tokens.PagedCache, B.int8t_cache_attend_division, B.int8t_cache_attend))
    cache = kind.empty(2 * pages, page, heads, dim, DEV)
    g = torch.Generator().manual_seed(1)
    n = 6000
    k, v, q = (torch.randn(m, h, dim, generator=g).to(dtype).to(DEV) for m, h in ((2 * n, heads), (2 * n, heads), (T, heads * group)))
    lengths = torch.tensor([n, n - 50], dtype=torch.int32, device=DEV)
    table = torch.arange(2 * pages, dtype=torch.int32, device=DEV).view(2, pages)
    at = torch.arange(n, device=DEV)
    cache.write(k, v, torch.cat([at, pages * page + at]))
    first = torch.tensor(starts, dtype=torch.int32, device=DEV)
    d = B.AttendDesc(T, 2, group, pages, 0, B.BF16, 1, dim ** -0.5, q.stride(0), q.stride(1), pages)
    how = divide(cache._c, d)
    assert how.shares > 1 and how.rows == rows
    ws = torch.full((cache._calls[2](cache._c, d) // 4,), float("nan"), device=DEV)
    out, lse = torch.full((T, heads * group, dim), 7.0, dtype=dtype, device=DEV), torch.full((T, heads * group), 7.0, device=DEV)
    attend(cache._c, d, q, first, lengths, table, out, lse, ws)
    own = torch.zeros(T, dtype=torch.bool, device=DEV)
    own[starts[0]:starts[-1]] = True
    assert (out[~own] == 7.0).all() and (lse[~own] == 7.0).all()
    # The others' are those of a call without such tokens, whose keys may be dealt out otherwise: either is off by half a step of bf16, by 2^-11 of the mean of |v|
    # (below 1) for the rounding of p and by less than that for the scores (2^-17 of their terms, some 7 together, twice).
    if own.any():
        want, wlse = cache.attend(q[own], first - starts[0], lengths, table, return_lse=True)
        assert torch.allclose(out[own].float(), want.float(), rtol=2.0**-7, atol=2.0**-9) and torch.allclose(lse[own], wlse, rtol=2.0**-18, atol=2.0**-12)
