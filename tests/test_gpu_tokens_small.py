"""Stochastic codes of rows and columns whose largest value is so small that 2^24 times its reciprocal passes fp32's range."""
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
from test_gpu_tokens import codes, pad16, same, unpad, values  # noqa: E402

DEV = torch.device("cuda:0")
F32, BF16 = torch.float32, torch.bfloat16


# 127 2^24 / 2^128 is 6.3e-30; beside it rows of ordinary size, which share their launch's blocks and columns their tiles
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(6, 70), (9, 1500), (5, 9000), (3, 33001), (130, 70)])
@pytest.mark.parametrize("size", [1e-28, 6e-30, 1e-30, 1e-33, 3e-36])
def test_codes(dtype, rows, cols, size):
    x, _ = values((rows, cols), 1)
    by_row, by_col = torch.ones(rows, 1), torch.ones(1, cols)
    by_row[::2], by_col[:, ::3] = size, size
    seed = 77
    for small, axis in ((by_row, 1), (by_col, 0)):
        v = (x / x.abs().amax(axis, keepdim=True) * small).to(dtype)
        want, scale = codes(v.float().numpy(), axis, seed)
        n, m = (rows, cols) if axis == 1 else (cols, rows)
        q, s = torch.full((n, pad16(m)), 99, dtype=torch.int8, device=DEV), torch.full((n,), -1.0, device=DEV)
        if axis == 1:
            B.int8t_quantize_rows(v.to(DEV), rows, cols, cols, None, B.ROUND_STOCHASTIC, seed, q, s, type=B.DTYPES[dtype])
        else:
            ws = torch.empty(B.int8t_quantize_cols_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
            B.int8t_quantize_cols(v.to(DEV), rows, cols, cols, None, B.ROUND_STOCHASTIC, seed, q, s, None, ws, type=B.DTYPES[dtype])
        assert np.array_equal(unpad(q, m), want if axis == 1 else want.T)
        assert np.array_equal(s.cpu().numpy(), scale.reshape(-1))


@pytest.mark.parametrize("M,K,N", [(40, 64, 72), (33, 48, 9001)])
def test_gradients(M, K, N):
    (x, x32), (w, w32), (g, _) = values((M, K), 2), values((N, K), 3), values((M, N), 4)
    g = g * 1e-31
    x, w = x.to(DEV).requires_grad_(True), w.to(DEV).requires_grad_(True)
    dx, dw = torch.autograd.grad(tokens.linear(x, w, seed=5), [x, w], g.to(DEV))
    (xq, sx), (wq, sw), g32 = codes(x32, 1), codes(w32, 1), g.numpy()
    gq, sg = codes(g32 * sw.T, 1, 5)
    hq, sh = codes(g32 * sx, 0, 5 ^ (1 << 63))
    same(dx, (gq @ wq).astype(np.float32) * sg, F32)
    same(dw, (hq.T @ xq).astype(np.float32) * sh.T, F32)
