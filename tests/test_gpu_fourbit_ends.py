"""4-bit codes drawn, and products of codes, where scales are at the ends of their range (2^-127, of which there is no normal fp32 number, to 2^126)."""
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
from test_gpu_fourbit_codes import check, quantise  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_drawn_codes(dtype):
    r = np.random.default_rng(1)
    x = np.concatenate([r.standard_normal((3, 300)) * 2.0**e for e in (-148, -140, -127, -126, -124, -100, 0, 100, 120, 124)]).astype(np.float32)
    x[-1, :5] = np.finfo(np.float32).max, -np.finfo(np.float32).max, 1e-45, 3e38, 2.0**127
    if dtype is BF16:
        x[-1, :2] = 2.0**127 * 1.9921875
    t = torch.from_numpy(x).to(dtype)
    assert torch.isfinite(t).all()
    x64, seed = t.double().numpy(), 1234567890123
    rows, cols = x64.shape
    index = np.arange(rows * cols).reshape(rows, cols)
    by_rows, by_cols, _ = quantise(t.to(DEV), rows, cols, cols, dtype, True, seed, sums=False)
    check(by_rows, x64, cols, R.draws(index, seed))
    check(by_cols, x64.T, rows, R.draws(index, seed ^ (1 << 63)).T)


@pytest.mark.parametrize("low", [True, False])
@pytest.mark.parametrize("M,N,K", [(16, 40, 256), (130, 70, 300), (300, 8200, 600), (1003, 4100, 70)])
def test_products(M, N, K, low):
    """Scales of 2^-127 to 2^-125 against 2^124 to 2^126: sums of products in steps of 2^-5, exact in fp32."""
    r = np.random.default_rng(2)

    def operand(rows, small):
        code = r.integers(0, 16, (rows, 32 * R.blocks_of(K)))
        code[:, K:] = 0
        byte = r.integers(0, 3, (rows, R.blocks_of(K))) if small else r.integers(251, 254, (rows, R.blocks_of(K)))
        return torch.from_numpy(R.packed(code)).to(DEV), torch.from_numpy(R.in_panels(byte, K)).to(DEV), torch.from_numpy(R.stands_for(code, byte, K)).to(DEV)
    (a, sa, av), (b, sb, bv) = operand(M, low), operand(N, not low)
    y = torch.empty(M, N, device=DEV)
    B.int8t_mx4_product(a, sa, b, sb, M, N, K, None, y, N)
    want = av @ bv.T.contiguous()
    assert float((av.abs() @ bv.abs().T.contiguous()).max()) * 2**5 < 2**24
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("M", [1, 9, 40])
@pytest.mark.parametrize("x_power,w_power", [(-126, 120), (-128, 125), (120, -120), (125, -128)])
def test_layers(M, x_power, w_power):
    """Each of the additions rounds (or cuts) by 2^-23 of what is summed at most, the result by half a step, below the normal numbers by half of 2^-149."""
    r, K, N = np.random.default_rng(3), 330, 50
    x = torch.from_numpy((r.standard_normal((M, K)) * 2.0**x_power).astype(np.float32))
    w = torch.from_numpy((r.standard_normal((N, K)) * 2.0**w_power).astype(np.float32))
    y = fourbit.ServedLinear4.of(w.to(DEV))(x.to(DEV)).double().cpu().numpy()
    a, b = R.rounded(x.double().numpy()), R.rounded(w.double().numpy())
    want, size = a @ b.T, np.abs(a) @ np.abs(b).T
    assert size.max() > 0 and (np.abs(y - want) <= (K + 1) * 2.0**-23 * size + 2.0**-24 * np.abs(want) + 2.0**-150).all()
