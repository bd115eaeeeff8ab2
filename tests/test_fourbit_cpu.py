"""Host side of the microscaled 4-bit operators, rotary positions and page tables, without a GPU: sizes, argument checks before any launch, refusals of the modules,
and the reference that the GPU tests go by."""
import ctypes as C
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import fourbit_reference as R  # noqa: E402
from paper_1912_12607_amd import binding as B  # noqa: E402
from paper_1912_12607_amd import fourbit, positions  # noqa: E402

FAKE, ODD, OFF4 = 0x10000, 0x10001, 0x10004          # addresses that these paths never follow
OTHER = 0x20000
BIG = 1 << 40
NULL, SHAPE, ARG, WORKSPACE = 1, 2, 3, 4


def call(name, *args):
    return getattr(B.lib, name)(*args)


def test_reference_codes():
    """A few by hand: 6 stays, 6.1 takes the next power of two, ties go to the even code."""
    x = np.zeros((1, 32))
    x[0, :9] = [6.0, 0.25, 0.75, -1.25, 1.75, 2.5, 3.5, 5.0, -0.0]
    code, byte = R.quantise(x)
    assert byte.tolist() == [[127]] and code[0, :9].tolist() == [7, 0, 2, 8 + 2, 4, 4, 6, 6, 8]
    x[0, 0] = 6.1
    code, byte = R.quantise(x)
    assert byte.tolist() == [[128]] and code[0, :3].tolist() == [5, 0, 1]
    assert R.quantise(np.full((1, 5), np.nan))[1].tolist() == [[255]] and R.quantise(np.zeros((1, 33)))[1].tolist() == [[0, 0]]
    assert np.array_equal(R.unpacked(R.packed(code)), code)
    # a draw of all ones goes up from anything that is not a level, one of all zeros never
    x[0, 0] = 6.0
    up, down = (R.quantise(x, np.full((1, 32), u))[0] & 7 for u in ((1 << 24) - 1, 0))
    assert up[0, :9].tolist() == [7, 1, 2, 3, 4, 5, 6, 7, 0] and down[0, :9].tolist() == [7, 0, 1, 2, 3, 4, 5, 6, 0]


def test_quantize_arguments():
    def go(x=FAKE, t=0, rows=4, cols=40, pitch=40, mode=0, q=FAKE, s=FAKE, qt=FAKE, st=FAKE, sums=FAKE, ws=FAKE, nb=BIG):
        return call("int8t_mx4_quantize", x, t, rows, cols, pitch, mode, 0, q, s, qt, st, sums, ws, nb, None)
    for bad in (dict(x=None), dict(q=None), dict(s=None), dict(qt=None), dict(st=None), dict(ws=None), dict(q=None, s=None, qt=None, st=None, sums=None)):
        assert go(**bad) == NULL, bad
    for bad in (dict(rows=0), dict(cols=0), dict(rows=-1), dict(pitch=39), dict(cols=B.MAX_REDUCTION + 1, pitch=1 << 20), dict(rows=B.MAX_REDUCTION + 1), dict(rows=1 << 20, cols=1 << 12, pitch=1 << 12)):
        assert go(**bad) == SHAPE, bad
    for bad in (dict(t=3), dict(mode=2), dict(x=ODD), dict(t=1, x=ODD), dict(q=OFF4), dict(s=OFF4), dict(qt=OFF4), dict(st=OFF4), dict(sums=ODD), dict(ws=OFF4)):
        assert go(**bad) == ARG, bad
    need = B.int8t_mx4_quantize_workspace_bytes(4, 40)
    assert need >= 160 and go(nb=need - 1) == WORKSPACE
    assert B.int8t_mx4_quantize_workspace_bytes(0, 4) == 0 and B.int8t_mx4_quantize_workspace_bytes(4, 0) == 0


def test_product_arguments():
    def go(a=FAKE, sa=FAKE, b=FAKE, sb=FAKE, M=4, N=5, K=33, bias=None, y=FAKE, t=0, pitch=5, ws=None, nb=0):
        return call("int8t_mx4_product", a, sa, b, sb, M, N, K, bias, y, t, pitch, ws, nb, None)
    for arg in ("a", "sa", "b", "sb", "y"):
        assert go(**{arg: None}) == NULL
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(K=B.MAX_REDUCTION + 1), dict(pitch=4), dict(M=1 << 23, N=1 << 23, pitch=1 << 23)):
        assert go(**bad) == SHAPE, bad
    for bad in (dict(t=-1), dict(t=7), dict(a=OFF4), dict(b=OFF4), dict(sa=OFF4), dict(sb=OFF4), dict(bias=ODD), dict(y=ODD), dict(ws=OFF4)):
        assert go(**bad) == ARG, bad
    assert B.int8t_mx4_product_workspace_bytes(4, 4, B.MAX_REDUCTION + 1) == 0
    out = B.Division()
    assert call("int8t_mx4_product_division", 4, 4, 32, 0, None) == NULL and call("int8t_mx4_product_division", 0, 4, 32, 0, C.byref(out)) == SHAPE
    assert B.int8t_mx4_product_division(8192, 4096, 4096).rows == 256 and B.int8t_mx4_product_division(8192, 4096, 4096).shares == 1


@pytest.mark.parametrize("backward", [0, 1])
def test_linear_arguments(backward):
    def go(d=(40, 64, 48, 0, 0), **changes):
        fields = dict(x=FAKE, w=FAKE, dy=FAKE, x_pitch=64, w_pitch=64, y_pitch=48, dy_pitch=48, wq=FAKE, sw=FAKE, wt=FAKE, swt=FAKE, xt=FAKE, sxt=FAKE, bias=None, y=FAKE,
                      dx=FAKE, dw=FAKE, db=None, ws=FAKE, ws_bytes=BIG)
        fields.update(changes)
        desc = None if d is None else B.LinearDesc(*d)
        args = (None if desc is None else C.byref(desc), C.byref(B.Mx4LinearBuffers(**fields))) + ((7,) if backward else ()) + (None,)
        return call("int8t_mx4_linear_bwd" if backward else "int8t_mx4_linear_fwd", *args)
    assert go(None) == NULL
    for d in ((-1, 64, 48, 0, 0), (40, 0, 48, 0, 0), (40, 64, 0, 0, 0), (40, B.MAX_REDUCTION + 1, 48, 0, 0), (1 << 20, 4096, 48, 0, 0)) + (
            ((0, 64, 48, 0, 0), (B.MAX_REDUCTION + 1, 64, 48, 0, 0), (40, 64, B.MAX_REDUCTION + 1, 0, 0)) if backward else ()):
        assert go(d) == SHAPE, d
        assert B.int8t_mx4_linear_workspace_bytes(B.LinearDesc(*d), backward) == 0
    for d in ((40, 64, 48, 3, 0), (40, 64, 48, 0, -1)):
        assert go(d) == ARG
    need = B.int8t_mx4_linear_workspace_bytes(B.LinearDesc(40, 64, 48, 0, 0), backward)
    assert need > 0 and go(ws_bytes=need - 1) == WORKSPACE
    if backward:
        for bad in (dict(dy=None), dict(ws=None), dict(dx=None, dw=None), dict(wt=None), dict(swt=None), dict(xt=None), dict(sxt=None)):
            assert go(**bad) == NULL, bad
        assert go(dy_pitch=47) == SHAPE
        for bad in (dict(dy=ODD), dict(dx=ODD), dict(dw=ODD), dict(db=ODD), dict(wt=OFF4), dict(swt=OFF4), dict(xt=OFF4), dict(sxt=OFF4), dict(ws=OFF4)):
            assert go(**bad) == ARG, bad
    else:
        for bad in (dict(x=None), dict(y=None), dict(wq=None), dict(sw=None), dict(wt=None), dict(sxt=None), dict(ws=None), dict(w=None), dict(w=None, wt=None, swt=None, wq=None, sw=None)):
            assert go(**bad) == NULL, bad
        for bad in (dict(x_pitch=63), dict(w_pitch=63), dict(y_pitch=47)):
            assert go(**bad) == SHAPE, bad
        for bad in (dict(x=ODD), dict(w=ODD), dict(y=ODD), dict(bias=ODD), dict(wq=OFF4), dict(sw=OFF4), dict(xt=OFF4), dict(swt=OFF4), dict(ws=OFF4)):
            assert go(**bad) == ARG, bad
        assert go((0, 64, 48, 0, 0), w=None, wt=None, swt=None) == 0           # no tokens, nothing to launch
        assert B.int8t_mx4_linear_workspace_bytes(B.LinearDesc(1, 4096, 48, 0, 0), 2) == 0 and B.int8t_mx4_linear_workspace_bytes(B.LinearDesc(1, 64, 48, 0, 0), 3) == 0


def cache(**changes):
    fields = dict(kq=FAKE, vq=FAKE, ks=FAKE, vs=FAKE, pages=10, page_size=16, heads=2, dim=64)
    fields.update(changes)
    return B.Mx4Cache(**fields)


@pytest.mark.parametrize("bad,status", [(dict(kq=None), NULL), (dict(vs=None), NULL), (dict(pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(heads=0), SHAPE), (dict(dim=0), SHAPE),
                                        (dict(dim=72), SHAPE), (dict(dim=272), SHAPE), (dict(pages=1 << 27), SHAPE), (dict(heads=65536), SHAPE), (dict(kq=OFF4), ARG), (dict(ks=OFF4), ARG)])
def test_cache_is_checked_by_every_call(bad, status):
    c, d = cache(**bad), B.AttendDesc(4, 2, 3, 8, 0, 0, 1, 0.125, 384, 64, 8)
    assert call("int8t_mx4_cache_write", C.byref(c), FAKE, FAKE, 0, 4, 128, 64, 128, 64, FAKE, None) == status
    assert call("int8t_mx4_cache_read", C.byref(c), FAKE, 4, FAKE, FAKE, 0, None) == status
    assert call("int8t_mx4_cache_attend", C.byref(c), C.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, BIG, None) == status
    assert call("int8t_mx4_cache_attend_workspace_bytes", C.byref(c), C.byref(d)) == 0
    assert call("int8t_mx4_cache_attend_division", C.byref(c), C.byref(d), C.byref(B.Division())) == status


def test_cache_move_and_attend_arguments():
    c = cache()

    def write(k=FAKE, v=FAKE, t=0, n=4, slots=FAKE):
        return call("int8t_mx4_cache_write", C.byref(c), k, v, t, n, 128, 64, 128, 64, slots, None)

    def read(k=FAKE, v=FAKE, t=0, n=4, slots=FAKE):
        return call("int8t_mx4_cache_read", C.byref(c), slots, n, k, v, t, None)
    for go in (write, read):
        for arg in ("k", "v", "slots"):
            assert go(**{arg: None}) == NULL
        assert go(n=-1) == SHAPE and go(n=1 << 30) == SHAPE and go(t=3) == ARG and go(k=ODD) == ARG and go(v=ODD) == ARG and go(slots=OFF4) == ARG
        assert go(n=0, k=None) == 0
    names = [f[0] for f in B.AttendDesc._fields_]

    def attend(q=FAKE, starts=FAKE, lengths=FAKE, table=FAKE, out=FAKE, lse=None, ws=FAKE, nb=BIG, **changes):
        f = dict(tokens=4, requests=2, group=3, table_width=8, longest=0, type=0, causal=1, scale=0.125, q_token_pitch=384, q_head_pitch=64, table_pitch=8)
        f.update(changes)
        return call("int8t_mx4_cache_attend", C.byref(c), C.byref(B.AttendDesc(*[f[n] for n in names])), q, starts, lengths, table, out, lse, ws, nb, None)
    for arg in ("q", "starts", "lengths", "table", "out"):
        assert attend(**{arg: None}) == NULL, arg
    for bad in (dict(tokens=-1), dict(requests=0), dict(group=0), dict(table_width=-1), dict(table_pitch=7), dict(tokens=1 << 29), dict(table_width=1 << 28, table_pitch=1 << 28)):
        assert attend(**bad) == SHAPE, bad
    for bad in (dict(type=3), dict(causal=2), dict(scale=math.inf), dict(q=ODD), dict(out=OFF4), dict(lse=ODD), dict(ws=OFF4)):
        assert attend(**bad) == ARG, bad
    long = dict(table_width=4096, table_pitch=4096)
    assert attend(nb=16, **long) == WORKSPACE and attend(ws=None, nb=0, **long) == NULL and attend(tokens=0, q=None) == 0


def test_rotate_arguments():
    def tensor(**changes):
        f = dict(x=FAKE, y=OTHER, x_token_pitch=128, x_head_pitch=64, y_token_pitch=128, y_head_pitch=64, heads=2)
        f.update(changes)
        return B.RotateTensor(**f)

    def go(first=tensor(), second=tensor(), positions=FAKE, turns=FAKE, **changes):
        f = dict(tokens=4, dim=64, rot=32, type=0, interleaved=0, back=0, amplitude=1.0)
        f.update(changes)
        return call("int8t_rotate", C.byref(B.RotateDesc(**f)), first if first is None else C.byref(first), second if second is None else C.byref(second), positions, turns, None)
    assert go(first=None) == NULL and go(first=tensor(x=None)) == NULL and go(second=tensor(y=None)) == NULL and go(positions=None) == NULL and go(turns=None) == NULL
    for bad in (dict(tokens=-1), dict(dim=0), dict(rot=0), dict(rot=33), dict(rot=66), dict(first=tensor(heads=0)), dict(first=tensor(heads=-1)), dict(second=tensor(heads=-1)), dict(tokens=1 << 30)):
        assert go(**bad) == SHAPE, bad
    for bad in (dict(type=3), dict(interleaved=2), dict(back=-1), dict(amplitude=math.nan), dict(amplitude=math.inf), dict(first=tensor(x=ODD)), dict(second=tensor(y=ODD)),
                dict(positions=ODD), dict(turns=OFF4), dict(first=tensor(y=FAKE, y_head_pitch=128))):
        assert go(**bad) == ARG, bad
    assert go(tokens=0, positions=None) == 0


def test_pages_arguments():
    def desc(**changes):
        f = dict(requests=2, width=4, page_size=16, pages=8, tokens=5, table_pitch=4)
        f.update(changes)
        return B.PagesDesc(**f)
    names = ["have", "add", "table", "free", "available", "lengths", "left", "starts", "slots", "positions", "without"]

    def extend(d=desc(), **changes):
        f = {n: 0x1000 * (i + 1) for i, n in enumerate(names)}
        f.update(changes)
        return call("int8t_pages_extend", d if d is None else C.byref(d), *[f[n] for n in names], None)

    def shrink(d=desc(), **changes):
        f = {n: 0x1000 * (i + 1) for i, n in enumerate(("stay", "lengths", "table", "free", "available"))}
        f.update(changes)
        return call("int8t_pages_shrink", d if d is None else C.byref(d), *[f[n] for n in ("stay", "lengths", "table", "free", "available")], None)
    for go, all_names in ((extend, names), (shrink, ["stay", "lengths", "table", "free", "available"])):
        assert go(None) == NULL
        for n in all_names:
            assert go(**{n: None}) == NULL, n
            assert go(**{n: ODD}) == ARG, n
        for bad in (dict(requests=-1), dict(width=-1), dict(page_size=0), dict(pages=-1), dict(tokens=-1), dict(tokens=2**31 - 1), dict(table_pitch=3), dict(width=1 << 28, table_pitch=1 << 28)):
            assert go(desc(**bad)) == SHAPE, bad
    assert extend(slots=0x9004) == ARG and extend(lengths=0x1000) == ARG and extend(lengths=0x2000) == ARG and extend(left=0x5000) == ARG


def test_host_tensors_and_bad_modules_are_refused():
    x, w = torch.zeros(2, 32), torch.zeros(4, 32)
    with pytest.raises(RuntimeError, match="device"):
        fourbit.linear4(x, w)
    with pytest.raises(RuntimeError):
        fourbit.ServedLinear4(torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8), 32)
    with pytest.raises(RuntimeError):
        fourbit.PagedCache4.empty(2, 16, 2, 64, "cpu")
    with pytest.raises(RuntimeError, match="device"):
        positions.Rotary(16)(torch.zeros(2, 3, 16), None, torch.zeros(2, dtype=torch.int32))
    with pytest.raises(RuntimeError, match="device"):
        positions.PageTable.empty(2, 3, 4, 16, "cpu")
    for bad in (dict(rot=7), dict(rot=0), dict(rot=8, layout="both"), dict(rot=8, base=0.0), dict(rot=8, factor=-1.0), dict(rot=8, original=10, slow=4.0, fast=2.0), dict(rot=8, frequencies=[1.0]),
                dict(rot=8, amplitude=math.inf)):
        with pytest.raises(ValueError):
            positions.Rotary(**bad)


def test_rotary_frequencies():
    r = positions.Rotary(8, base=100.0)
    assert torch.allclose(r.frequencies, torch.tensor([1.0, 100.0**-0.25, 0.1, 100.0**-0.75], dtype=torch.float64), rtol=1e-14)
    # 1000 positions: 159, 50, 15.9 and 5.03 turns
    r = positions.Rotary(8, base=100.0, factor=4.0, original=1000, slow=10.0, fast=100.0)
    turns = 1000 * 100.0**-0.25 / (2 * math.pi)
    keep = (turns - 10.0) / 90.0
    want = [1.0, 100.0**-0.25 * (keep + (1 - keep) / 4), 0.1 * ((1000 * 0.1 / (2 * math.pi) - 10) / 90 * 0.75 + 0.25), 100.0**-0.75 / 4]
    assert torch.allclose(r.frequencies, torch.tensor(want, dtype=torch.float64), rtol=1e-14)


def test_memory_shared_by_two_tensors():
    qkv = torch.zeros(5, 7, 16)
    assert not positions._share(qkv[:, :4], qkv[:, 4:6]) and positions._share(qkv[:, :5], qkv[:, 4:6]) and not positions._share(qkv[:2], qkv[2:4])
    assert positions._share(qkv[:3], qkv[2:5]) and not positions._share(qkv, torch.zeros(5, 7, 16))
    assert positions._overlaps(qkv[:, :1].expand(5, 3, 16)) and not positions._overlaps(qkv) and not positions._overlaps(qkv[:, 1::2]) and not positions._overlaps(qkv[::2])


def test_division_of_attention_at_the_edges():
    """Fewer tokens than requests, no pages, tables of the greatest length, blocks of every size: some division, scratch within 2^20 (dim + 2) bytes."""
    for dim in (16, 64, 96, 128, 256):
        for page in (1, 16, 24):
            c = cache(dim=dim, page_size=page, heads=8)
            for tokens in (1, 5, 63, 64, 700, 20000):
                for requests in (1, 3, 64, 600, 5000):
                    for group in (1, 7):
                        for width in (0, 1, 40, (2**31 - 5000) // page):
                            for kind, longest in ((B.F32, 0), (B.BF16, 1), (B.F16, 3000), (B.BF16, 2**31 - 1)):
                                d = B.AttendDesc(tokens, requests, group, width, longest, kind, 1, 0.1, 8 * group * dim, dim, width)
                                how, size = B.int8t_mx4_cache_attend_division(c, d), call("int8t_mx4_cache_attend_workspace_bytes", C.byref(c), C.byref(d))
                                assert how.rows in (16, 128, 256) and how.waves in (4, 8) and 1 <= how.shares <= 512
                                assert (size > 0) == (how.shares > 1) and size <= (2**20 + 4096) * (dim + 2) + 512
