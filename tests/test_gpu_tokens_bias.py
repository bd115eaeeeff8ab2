"""The bias's gradient without the weights': the library's own sums, the same as with them."""
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


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("M,K,N", [(1, 16, 1), (33, 48, 20), (2100, 64, 300), (40, 16, 9001)])
@pytest.mark.parametrize("want_x", [False, True])
def test_bias_without_weights(dtype, M, K, N, want_x):
    gen = torch.Generator().manual_seed(M)
    x, w, g = (torch.randn(*s, generator=gen).to(dtype).to(DEV) for s in ((M, K), (N, K), (M, N)))
    b = torch.randn(N, generator=gen).to(DEV).requires_grad_(True)

    def grads(*leaves):
        xs, ws = x.clone().requires_grad_("x" in leaves), w.clone().requires_grad_("w" in leaves)
        y = tokens.linear(xs, ws, b, seed=4)
        return torch.autograd.grad(y, [t for n, t in (("x", xs), ("w", ws), ("b", b)) if n in leaves], g)
    full = grads("x", "w", "b")
    B.int8t_profile_start(None)
    part = grads("x", "b") if want_x else grads("b")
    seen = B.int8t_profile_stop()
    assert torch.equal(part[-1], full[2]) and (not want_x or torch.equal(part[0], full[0]))
    assert seen["quantize_cols_kernel"][0] == 2
