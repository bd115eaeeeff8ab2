"""Products of 4-bit codes, and the layers through them, in each of their divisions: tiles of 64, 128 (two and three stages) and 256 rows, whole and split reductions, two products in one launch and in
two.  Each test asks the library for the division and asserts it.  All values are levels of the codes times powers of two that a tile of 32 x 32 shares, so that codes along either axis
stand for them exactly (a draw moves no level), all sums are exact in fp32 in any order, and results are equal to those in 64 bits, rounded once."""
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
from paper_1912_12607_amd import fourbit  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def exact(rows, cols, seed, dtype=F32):
    g = torch.Generator(device=DEV).manual_seed(seed)
    level = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)[torch.randint(0, 8, (rows, cols), generator=g, device=DEV)]
    sign = torch.randint(0, 2, (rows, cols), generator=g, device=DEV) * 2.0 - 1.0
    power = 2.0 ** torch.randint(-1, 2, (-(-rows // 32), -(-cols // 32)), generator=g, device=DEV)
    return (level * sign * power.repeat_interleave(32, 0)[:rows].repeat_interleave(32, 1)[:, :cols]).to(dtype)


def matmul(a, b, bias=None, dtype=F32):
    """a b^T + bias as the kernels round it; sums in steps of 2^-4 stay below 2^20, so that fp32 holds them all."""
    a, b = a.double(), b.double()
    assert float((a.abs() @ b.abs().T.contiguous()).max()) < 2.0**20
    y = (a @ b.T.contiguous()).float()
    return (y if bias is None else y + bias).to(dtype)


def division(M, N, K, scratch=True):
    d = B.int8t_mx4_product_division(M, N, K, B.int8t_mx4_product_workspace_bytes(M, N, K) if scratch else 0)
    return d.rows, d.stages, d.shares


def codes(x):
    rows, cols = x.shape
    q = torch.empty(rows, 16 * -(-cols // 32), dtype=torch.uint8, device=DEV)
    s = torch.empty(-(-cols // 256), rows, 8, dtype=torch.uint8, device=DEV)
    B.int8t_mx4_quantize(x, rows, cols, cols, B.ROUND_NEAREST_EVEN, 0, q, s, type=B.F32)
    return q, s


PRODUCTS = [(300, 257, 600, (64, 4, 1)), (385, 8203, 300, (128, 2, 1)), (200, 8203, 300, (128, 3, 1)), (257, 16385, 600, (128, 2, 1)), (1003, 8201, 70, (256, 2, 1)), (2001, 4097, 300, (256, 2, 1)),
            (17, 515, 16400, (64, 4, 8)), (1, 33, 8200, (64, 4, 8)), (300, 257, 16400, (64, 4, 4)), (17, 8203, 16400, (64, 4, 2))]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("M,N,K,how", PRODUCTS)
def test_products(M, N, K, how, bias, dtype):
    assert division(M, N, K) == how
    a, b, c = exact(M, K, 1), exact(N, K, 2), torch.randn(N, generator=torch.Generator(device=DEV).manual_seed(3), device=DEV) if bias else None
    (aq, sa), (bq, sb) = codes(a), codes(b)
    want = matmul(a, b, c, dtype)
    # rows that 16-byte stores take, whose last piece they do not fill, and others
    for pitch in (N, (N + 15) & ~7, N + 3):
        for scratch in (True, False):
            size = B.int8t_mx4_product_workspace_bytes(M, N, K)
            assert (size > 0) == (how[2] > 1) and division(M, N, K, False)[2] == 1
            if not scratch and not size:
                continue
            y = torch.full((M + 1, pitch), 3.0, dtype=dtype, device=DEV)
            ws = torch.full((size // 4,), float("nan"), device=DEV) if scratch and size else None
            B.int8t_mx4_product(aq, sa, bq, sb, M, N, K, c, y, pitch, type=B.DTYPES[dtype], ws=ws)
            assert torch.equal(y[:M, :N], want) and (y[M] == 3.0).all() and (y[:, N:] == 3.0).all()


LAYERS = [(70, 16400, 70, (128, 3, 1), (128, 3, 1)), (130, 16400, 130, (128, 2, 1), (128, 2, 1)), (385, 16400, 385, (256, 2, 1), (256, 2, 1)), (8200, 17, 17, (64, 4, 1), (64, 4, 8)),
          (17, 17, 8200, (64, 4, 8), (64, 4, 1)), (16400, 257, 300, (128, 2, 1), (64, 4, 4)), (130, 700, 16400, (64, 4, 4), (256, 2, 1)), (16400, 385, 17, (256, 2, 1), (64, 4, 8)),
          (17, 16400, 70, (64, 4, 1), (128, 3, 1)), (513, 200, 40, (64, 4, 1), (64, 4, 1))]


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, BF16), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("M,K,N,of_x,of_w", LAYERS)
def test_layers_and_their_gradients(M, K, N, of_x, of_w, dtype, wtype):
    assert division(M, K, N) == of_x and division(N, K, M) == of_w
    x, w, g = exact(M, K, 1, dtype), exact(N, K, 2, wtype), exact(M, N, 3, dtype)
    b = torch.randn(N, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV)
    y, dx, dw, db = (matmul(x, w, b, dtype), matmul(g, w.T.contiguous(), None, dtype), matmul(g.T.contiguous(), x.T.contiguous(), None, wtype), g.double().sum(0).float())
    for wanted in ((0, 1, 2), (0, 1), (1, 2), (0, 2), (2,)):
        leaves = [t.clone().requires_grad_(i in wanted) for i, t in enumerate((x, w, b))]
        out = fourbit.linear4(*leaves, seed=77)
        assert torch.equal(out, y)
        got = torch.autograd.grad(out, [leaves[i] for i in wanted], g)
        for i, t in zip(wanted, got):
            assert torch.equal(t, (dx, dw, db)[i]), "x w b".split()[i]
    assert torch.equal(fourbit.ServedLinear4.of(w, b)(x), y)
