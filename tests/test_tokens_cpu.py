"""Host side of the token operators, without a GPU: sizes, argument checks before any launch, refusals of the modules."""
import ctypes as C
import math

import pytest

torch = pytest.importorskip("torch")

from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import tokens  # noqa: E402

FAKE, ODD, OFF4 = 0x10000, 0x10001, 0x10004          # addresses that these paths never follow
BIG = 1 << 40
NULL, SHAPE, ARG, WORKSPACE = 1, 2, 3, 4


def call(name, *args):
    return getattr(B.lib, name)(*args)


@pytest.mark.parametrize("name", ["int8t_quantize_rows", "int8t_quantize_cols"])
def test_quantize_arguments(name):
    cols = name.endswith("cols")

    def go(x=FAKE, t=0, rows=4, cols_=40, pitch=40, f=None, mode=0, q=FAKE, s=FAKE, sums=None, ws=FAKE, nb=BIG):
        return call(name, x, t, rows, cols_, pitch, f, mode, 0, q, s, *((sums, ws, nb) if cols else ()), None)
    for arg in ("x", "q", "s") + (("ws",) if cols else ()):
        assert go(**{arg: None}) == NULL
    for bad in (dict(rows=0), dict(cols_=0), dict(rows=-1), dict(pitch=39), dict(rows=1 << 20, cols_=1 << 12, pitch=1 << 12)):
        assert go(**bad) == SHAPE
    for bad in (dict(t=3), dict(mode=2), dict(x=ODD), dict(t=1, x=ODD), dict(q=OFF4), dict(s=OFF4)):
        assert go(**bad) == ARG
    if cols:
        assert go(nb=16) == WORKSPACE and go(ws=OFF4) == ARG and go(sums=ODD) == ARG
        assert B.int8t_quantize_cols_workspace_bytes(0, 4) == 0 and B.int8t_quantize_cols_workspace_bytes(1000, 300) >= 2 * 300 * 4
    else:
        assert go(f=OFF4) == ARG


def test_transpose_and_product_arguments():
    assert call("int8t_transpose_codes", None, 4, 4, FAKE, None) == NULL
    assert call("int8t_transpose_codes", FAKE, 0, 4, FAKE, None) == SHAPE
    assert call("int8t_transpose_codes", FAKE, 4, 4, OFF4, None) == ARG

    def go(a=FAKE, sa=FAKE, b=FAKE, sb=None, M=4, N=5, K=33, bias=None, y=FAKE, t=0, pitch=5, ws=None, nb=0):
        return call("int8t_product", a, sa, b, sb, M, N, K, bias, y, t, pitch, ws, nb, None)
    for arg in ("a", "sa", "b", "y"):
        assert go(**{arg: None}) == NULL
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(K=B.MAX_REDUCTION + 1), dict(pitch=4)):
        assert go(**bad) == SHAPE
    for bad in (dict(t=-1), dict(t=7), dict(a=OFF4), dict(b=OFF4), dict(sa=ODD), dict(sb=ODD), dict(bias=ODD), dict(y=ODD), dict(ws=OFF4)):
        assert go(**bad) == ARG
    assert B.int8t_product_workspace_bytes(4, 4, B.MAX_REDUCTION + 1) == 0


def buffers(**changes):
    fields = dict(x=FAKE, w=FAKE, dy=FAKE, x_pitch=64, w_pitch=64, y_pitch=48, dy_pitch=48, xq=FAKE, wq=FAKE, sx=FAKE, sw=FAKE, bias=None, y=FAKE, dx=FAKE, dw=FAKE,
                  db=None, ws=FAKE, ws_bytes=BIG)
    fields.update(changes)
    return B.LinearBuffers(**fields)


@pytest.mark.parametrize("backward", [0, 1])
def test_linear_arguments(backward):
    def go(d=(8, 64, 48, 0, 0), **changes):
        desc, b = (None if d is None else B.LinearDesc(*d)), buffers(**changes)
        args = (None if desc is None else C.byref(desc), C.byref(b)) + ((7,) if backward else ()) + (None,)
        return call("int8t_linear_bwd" if backward else "int8t_linear_fwd", *args)
    assert go(None) == NULL
    for d in ((-1, 64, 48, 0, 0), (8, 0, 48, 0, 0), (8, 64, 0, 0, 0), (8, B.MAX_REDUCTION + 1, 48, 0, 0), (1 << 20, 4096, 48, 0, 0)) + (
            ((0, 64, 48, 0, 0), (B.MAX_REDUCTION + 1, 64, 48, 0, 0), (8, 64, B.MAX_REDUCTION + 1, 0, 0)) if backward else ()):
        assert go(d) == SHAPE, d
        assert B.int8t_linear_workspace_bytes(B.LinearDesc(*d), backward) == 0
    for d in ((8, 64, 48, 3, 0), (8, 64, 48, 0, -1)):
        assert go(d) == ARG
    need = B.int8t_linear_workspace_bytes(B.LinearDesc(8, 64, 48, 0, 0), backward)
    assert need > 0 and go(ws_bytes=need - 1) == WORKSPACE
    if backward:
        for bad in (dict(dy=None), dict(ws=None), dict(dx=None, dw=None), dict(wq=None), dict(sw=None), dict(xq=None), dict(sx=None)):
            assert go(**bad) == NULL, bad
        assert go(dy_pitch=47) == SHAPE
        for bad in (dict(dy=ODD), dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(wq=OFF4), dict(sw=OFF4), dict(xq=OFF4), dict(sx=OFF4), dict(ws=OFF4)):
            assert go(**bad) == ARG, bad
    else:
        for bad in (dict(x=None), dict(y=None), dict(wq=None), dict(sw=None), dict(ws=None), dict(xq=None), dict(sx=None)):
            assert go(**bad) == NULL, bad
        for bad in (dict(x_pitch=63), dict(w_pitch=63), dict(y_pitch=47)):
            assert go(**bad) == SHAPE, bad
        for bad in (dict(x=ODD), dict(w=ODD), dict(y=ODD), dict(bias=ODD), dict(wq=OFF4), dict(sw=OFF4), dict(xq=OFF4), dict(sx=OFF4), dict(ws=OFF4)):
            assert go(**bad) == ARG, bad
        assert go((0, 64, 48, 0, 0), w=None) == 0           # no tokens, nothing to launch


def cache(**changes):
    fields = dict(kq=FAKE, vq=FAKE, ks=FAKE, vs=FAKE, pages=10, page_size=16, heads=2, dim=64)
    fields.update(changes)
    return B.Cache(**fields)


BAD_CACHES = [(dict(kq=None), NULL), (dict(vs=None), NULL), (dict(pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(heads=0), SHAPE), (dict(dim=0), SHAPE),
              (dict(dim=72), SHAPE), (dict(dim=272), SHAPE), (dict(pages=1 << 27), SHAPE), (dict(heads=65536), SHAPE), (dict(kq=OFF4), ARG), (dict(ks=OFF4), ARG)]


@pytest.mark.parametrize("bad,status", BAD_CACHES)
def test_cache_is_checked_by_every_call(bad, status):
    c, d = cache(**bad), B.AttendDesc(4, 2, 3, 8, 0, 0, 1, 0.125, 384, 64, 8)
    assert call("int8t_cache_write", C.byref(c), FAKE, FAKE, 0, 4, 128, 64, 128, 64, FAKE, None) == status
    assert call("int8t_cache_read", C.byref(c), FAKE, 4, FAKE, FAKE, 0, None) == status
    assert call("int8t_cache_attend", C.byref(c), C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG, None) == status
    assert call("int8t_cache_attend_workspace_bytes", C.byref(c), C.byref(d)) == 0


def test_cache_move_arguments():
    c = cache()

    def write(k=FAKE, v=FAKE, t=0, n=4, slots=FAKE):
        return call("int8t_cache_write", C.byref(c), k, v, t, n, 128, 64, 128, 64, slots, None)

    def read(k=FAKE, v=FAKE, t=0, n=4, slots=FAKE):
        return call("int8t_cache_read", C.byref(c), slots, n, k, v, t, None)
    for go in (write, read):
        for arg in ("k", "v", "slots"):
            assert go(**{arg: None}) == NULL
        assert go(n=-1) == SHAPE and go(n=1 << 30) == SHAPE and go(t=3) == ARG and go(k=ODD) == ARG and go(v=ODD) == ARG and go(slots=OFF4) == ARG
        assert go(n=0, k=None) == 0
    assert call("int8t_cache_write", None, FAKE, FAKE, 0, 4, 128, 64, 128, 64, FAKE, None) == NULL


def test_attend_arguments():
    c = cache()
    names = [f[0] for f in B.AttendDesc._fields_]

    def desc(**changes):
        f = dict(tokens=4, requests=2, group=3, table_width=8, longest=0, type=0, causal=1, scale=0.125, q_token_pitch=384, q_head_pitch=64, table_pitch=8)
        f.update(changes)
        return B.AttendDesc(*[f[n] for n in names])

    def go(q=FAKE, starts=FAKE, lengths=FAKE, table=FAKE, out=FAKE, lse=None, ws=FAKE, nb=BIG, **changes):
        return call("int8t_cache_attend", C.byref(c), C.byref(desc(**changes)), q, starts, lengths, table, out, lse, ws, nb, None)
    for arg in ("q", "starts", "lengths", "table", "out"):
        assert go(**{arg: None}) == NULL, arg
    for bad in (dict(tokens=-1), dict(requests=-1), dict(requests=0), dict(group=0), dict(table_width=-1), dict(longest=-1), dict(table_pitch=7), dict(tokens=1 << 29),
                dict(table_width=1 << 28, table_pitch=1 << 28)):
        assert go(**bad) == SHAPE, bad
    for bad in (dict(type=3), dict(causal=2), dict(scale=math.inf), dict(scale=math.nan), dict(q=ODD), dict(starts=ODD), dict(lengths=ODD), dict(table=ODD), dict(out=OFF4),
                dict(lse=ODD), dict(ws=OFF4)):
        assert go(**bad) == ARG, bad
    long = dict(table_width=4096, table_pitch=4096)
    need = B.int8t_cache_attend_workspace_bytes(c, desc(**long))
    assert need > 0 and go(nb=need - 1, **long) == WORKSPACE and go(ws=None, nb=0, **long) == NULL
    assert B.int8t_cache_attend_workspace_bytes(c, desc(longest=64, **long)) == 0           # short contexts are not divided
    assert go(tokens=0, q=None) == 0


def test_attend_of_too_many_blocks():
    c = cache(heads=65535, dim=16, page_size=1)
    d = B.AttendDesc(4, 1 << 20, 1, 8, 0, 0, 1, 0.125, 16, 16, 8)
    assert call("int8t_cache_attend", C.byref(c), C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG, None) == SHAPE
    assert call("int8t_cache_attend_workspace_bytes", C.byref(c), C.byref(d)) == 0


def test_host_tensors_are_refused():
    x, w = torch.zeros(2, 32), torch.zeros(4, 32)
    with pytest.raises(RuntimeError, match="device"):
        tokens.linear(x, w)
    with pytest.raises(RuntimeError):
        tokens.ServedLinear(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4), 32)
    with pytest.raises(RuntimeError):
        tokens.PagedCache.empty(2, 16, 2, 64, "cpu")
