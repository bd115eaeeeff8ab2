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


def linear(M, K, N, w=None, xq=None, ws=FAKE):
    b = B.LinearBuffers(x=FAKE, w=w, x_pitch=K, w_pitch=K, y_pitch=N, xq=xq, wq=FAKE, sx=xq, sw=FAKE, y=FAKE, ws=ws, ws_bytes=BIG)
    return B.lib.int8t_linear_fwd(C.byref(B.LinearDesc(M, K, N, B.BF16, B.BF16)), C.byref(b), None)


# 2^32 threads and more in a launch: 64 at least for a row, 256 for a tile of 64 x 64 results
def test_launches_of_too_many_threads():
    most = (1 << 26) - 4
    assert B.lib.int8t_quantize_rows(FAKE, B.BF16, most + 1, 16, 16, None, 0, 0, FAKE, FAKE, None) == SHAPE
    assert linear(most + 1, 16, 5) == SHAPE                                 # served
    assert linear(most + 1, 16, 5, w=FAKE, xq=FAKE) == SHAPE                # kept for a backward pass
    assert linear(5, 16, most + 1, w=FAKE, xq=FAKE) == SHAPE                # as many output channels
    for M, N in ((1 << 26, 1 << 26), (1 << 20, 1 << 25)):
        assert B.lib.int8t_product(FAKE, FAKE, FAKE, FAKE, M, N, 16, None, FAKE, B.BF16, N, None, 0, None) == SHAPE


# pages of tiles ahead are looked up by places counted in an int: a table whose places nearly fill one is refused
@pytest.mark.parametrize("width,page,status", [((1 << 31) - 1, 1, SHAPE), ((1 << 27) - 1, 16, SHAPE), ((1 << 21) - 1, 1024, SHAPE),
                                               ((1 << 31) - 4096, 1, SHAPE), ((1 << 31) - 4097, 1, WORKSPACE)])
@pytest.mark.parametrize("tokens_", [1, 4000])
def test_tables_that_an_int_cannot_count(width, page, status, tokens_):
    c = B.Cache(FAKE, FAKE, FAKE, FAKE, 1, page, 1, 16)
    d = B.AttendDesc(tokens_, 1, 1, width, 0, B.BF16, 1, 0.25, 16, 16, width)
    need = B.int8t_cache_attend_workspace_bytes(c, d)
    assert (need > 0) == (status != SHAPE)
    assert B.lib.int8t_cache_attend(C.byref(c), C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, max(need, 1) - 1, None) == status


# shares of the keys go by a table's length, which may be many times the requests': what they leave for the joining pass stays within 2^14 blocks of 16 rows of dim
# sums, a maximum and a sum (2^20 (dim + 2) bytes), and blocks that fill the chip many times over are not divided at all
@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("kind", [B.F32, B.BF16])
@pytest.mark.parametrize("requests,new,heads,group", [(1, 1, 8, 4), (64, 1, 8, 4), (64, 95, 8, 4), (1, 12, 64, 1), (300, 1, 8, 8), (2000, 1, 8, 1), (5, 20, 32, 1)])
@pytest.mark.parametrize("width", [1, 100, 8192, 65536, 1 << 23])
def test_scratch_of_attention(requests, new, heads, group, dim, kind, width):
    c = B.Cache(FAKE, FAKE, FAKE, FAKE, 1 << 20, 16, heads, dim)
    need = [B.int8t_cache_attend_workspace_bytes(c, B.AttendDesc(requests * new, requests, group, width, longest, kind, 1, 0.125, dim, dim, width))
            for longest in (0, 1, 16 * width)]
    assert need[0] == need[2] and max(need) <= ((dim + 2) << 20) + 512
    if requests * new * group * heads >= 1 << 18:
        assert max(need) == 0


def test_divisions_are_asked_for_with_sizes_that_a_call_takes():
    out = B.Division()
    assert B.lib.int8t_product_division(8, 8, 8, 0, None) == NULL
    for bad in ((0, 8, 8), (8, 0, 8), (8, 8, 0), (8, 8, B.MAX_REDUCTION + 1), (1 << 26, 1 << 26, 16)):
        assert B.lib.int8t_product_division(*bad, 0, C.byref(out)) == SHAPE
    assert B.int8t_product_division(8, 8, 100000).shares == 1                # (no scratch)
    c, d = B.Cache(FAKE, FAKE, FAKE, FAKE, 10, 16, 2, 64), B.AttendDesc(4, 2, 3, 8, 0, 0, 1, 0.125, 384, 64, 8)
    assert B.lib.int8t_cache_attend_division(C.byref(c), C.byref(d), None) == NULL
    assert B.int8t_cache_attend_division(c, d).rows == 16
    d.tokens = 0
    assert B.lib.int8t_cache_attend_division(C.byref(c), C.byref(d), C.byref(out)) == SHAPE
    d.tokens, c.dim = 4, 65
    assert B.lib.int8t_cache_attend_division(C.byref(c), C.byref(d), C.byref(out)) == SHAPE
