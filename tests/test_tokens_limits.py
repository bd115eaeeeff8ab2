"""What the token operators refuse because their kernels cannot count so far; without a GPU, before any launch."""
import ctypes as C

import pytest

torch = pytest.importorskip("torch")

from paper_1912_12607_amd import binding as B  # noqa: E402

if torch.cuda.is_available():
    pytest.skip("addresses that no launch may follow", allow_module_level=True)

FAKE, BIG = 0x10000, 1 << 60
NULL, SHAPE, ARG, WORKSPACE = 1, 2, 3, 4


# rows beyond 32768 values are passed in steps of 32768 counted in an int: from 2^31 - 32768 on the count would not end
@pytest.mark.parametrize("cols", [(1 << 31) - 32767, (1 << 31) - 16])
def test_rows_that_a_loop_cannot_count(cols):
    assert B.lib.int8t_quantize_rows(FAKE, B.BF16, 1, cols, cols, None, 0, 0, FAKE, FAKE, None) == SHAPE
