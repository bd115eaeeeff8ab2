"""linear4 and its module where no graph records: the same results, nothing kept, and sizes that only a backward pass does not take."""
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

from paper_1912_12607_amd import fourbit  # noqa: E402

DEV = torch.device("cuda:0")
MODES = [torch.no_grad, torch.inference_mode]


def normal(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("M,K,N", [(131073, 1, 1), (3, 32, 151936)])
def test_sizes_that_only_a_backward_pass_does_not_take(mode, M, K, N):
    x, w, b = normal(M, K), normal(N, K, seed=1), normal(N, seed=2)
    want = fourbit.linear4(x, w, b)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    with pytest.raises(RuntimeError, match="not served"):
        fourbit.linear4(*leaves)
    with mode():
        assert torch.equal(fourbit.linear4(*leaves), want)


@pytest.mark.parametrize("mode", MODES)
@pytest.mark.parametrize("dtype,wdtype", [(torch.float32, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float32)])
@pytest.mark.parametrize("M", [0, 1, 77, 300])
def test_the_same_results(mode, dtype, wdtype, M):
    layer = fourbit.TokenLinear4(200, 90, dtype=wdtype, name="proj")
    x = normal(M, 200, dtype=dtype).requires_grad_(True)
    y = layer(x)
    assert y.requires_grad and y.shape == (M, 90)
    with mode():
        z = layer(x)
    assert not z.requires_grad and z.dtype is dtype and torch.equal(z, y)


@pytest.mark.parametrize("mode", MODES)
def test_nothing_is_kept(mode):
    """The memory that lives after a call is the result's alone, and at most the codes of one direction's lived within."""
    M, K, N = 512, 4096, 4096
    layer, x = fourbit.TokenLinear4(K, N, dtype=torch.bfloat16), normal(M, K, dtype=torch.bfloat16)
    with mode():
        y = layer(x)
        del y
        torch.cuda.synchronize()
        before = torch.cuda.memory_allocated()
        torch.cuda.reset_peak_memory_stats()
        y = layer(x)
        after, peak = torch.cuda.memory_allocated(), torch.cuda.max_memory_allocated()
    assert after - before == y.numel() * 2
    desc, (need, _, _), _, size = fourbit._plan(M, K, N, 1, 1)
    assert size > (M + N) * K // 2 and peak - before <= y.numel() * 2 + need + 4096
