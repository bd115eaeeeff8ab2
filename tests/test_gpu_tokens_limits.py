"""Calls of the token operators whose launches are larger than a dimension of a grid."""
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

from paper_1912_12607_amd import tokens  # noqa: E402

DEV = torch.device("cuda:0")


def test_cache_of_more_rows_than_a_grid_has_threads():
    """2^29 rows and some of eight lanes each: 2^32 threads and some.  The first and the last tokens have places, the others none."""
    heads, dim, n = 1024, 16, (1 << 19) + 3
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("needs 48 GiB")
    cache = tokens.PagedCache.empty(2, 4, heads, dim, DEV)
    row = torch.arange(1, dim + 1, device=DEV, dtype=torch.float16)
    k, v = row.expand(n, heads, dim), (-row).expand(n, heads, dim)
    slots = torch.full((n,), -1, dtype=torch.int64, device=DEV)
    slots[0], slots[n - 1], slots[n - 2] = 5, 1, 6
    cache.write(k, v, slots)
    there = torch.zeros(8, dtype=torch.bool, device=DEV)
    there[torch.tensor([5, 1, 6], device=DEV)] = True
    codes = (row.float() * (127.0 / 16)).round().to(torch.int8)
    for q, s, sign in ((cache.kq, cache.ks, 1), (cache.vq, cache.vs, -1)):
        q, s = q.transpose(1, 2).reshape(8, heads, dim), s.transpose(1, 2).reshape(8, heads)
        assert bool((q[there] == sign * codes).all()) and not q[~there].any()
        assert bool((s[there] == float(np.float32(16) / np.float32(127))).all()) and not s[~there].any()
    got = cache.read(slots, torch.float16)
    for t, want in zip(got, (codes * 1.0, codes * -1.0)):
        want = (want * cache.ks[1, 0, 1]).to(torch.float16)
        assert bool((t[[0, n - 1, n - 2]] == want).all()) and not t[1].any() and not t[n - 3].any()
