"""The attention layer of examples/: serving in chunks and single tokens gives what its parts give at once, training lowers the loss."""
import importlib.util
import os

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "attention_layer.py")
    spec = importlib.util.spec_from_file_location("attention_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


# Served: the projections of a token do not depend on its chunk (integer sums, the same epilogue), so the cache holds the same codes; what is left is
# attention's own error, bounded as for any p in two fp16 pieces by a unit roundoff of bf16 per output, the output's rounding (2^-8 of a value),
# whose effect through the last projection - nearest codes of its input, half a code or 1/254 of a token's maximum, in each of two roundings that may fall apart by one code,
# 1/127 - is at most |w| summed over the inputs times that.  The bound: (1/127 + 2^-7) max|input of o| sum|w_o|, far above what random signs give.
@pytest.mark.parametrize("heads,kv_heads,dim,lengths,chunk,singles", [(4, 2, 64, [70, 1, 33], 16, 5), (8, 1, 128, [150, 40], 150, 3), (3, 3, 16, [20, 19, 5, 1], 7, 20)])
def test_served_in_parts_and_at_once(heads, kv_heads, dim, lengths, chunk, singles):
    m = example()
    torch.manual_seed(3)
    layer = m.Attention(96, heads, kv_heads, dim)
    x = [torch.randn(n, 96, device="cuda:0").bfloat16() for n in lengths]
    with torch.no_grad():
        parts = m.serve(layer, x, chunk, singles)
        at_once = m.serve(layer, x, max(lengths), 0, page_size=24)
        # the layer's own parts, attention in 64 bits over what the cache holds
        q, k, v, o = (p.served() for p in (layer.q, layer.k, layer.v, layer.o))
        for t, y, z in zip(x, parts, at_once):
            n = t.shape[0]
            cache = m.PagedCache.empty(1, n, kv_heads, dim)
            slots = torch.arange(n, device="cuda:0")
            cache.write(k(t).view(n, kv_heads, dim), v(t).view(n, kv_heads, dim), slots)
            kk, vv = (c.double().cpu().repeat_interleave(heads // kv_heads, 1).transpose(0, 1).contiguous() for c in cache.read(slots))
            qq = q(t).view(n, heads, dim).double().cpu().transpose(0, 1)
            s = qq @ kk.transpose(1, 2) * dim ** -0.5
            s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), float("-inf"))
            a = (s.softmax(-1) @ vv).transpose(0, 1).reshape(n, -1)
            want = a @ layer.o.weight.double().cpu().t()
            bound = (1 / 127 + 2.0 ** -7) * a.abs().amax(1, keepdim=True) * layer.o.weight.double().cpu().abs().sum(1) \
                + (layer.o.weight.double().cpu().abs().amax(1) / 254) * a.abs().sum(1, keepdim=True) + want.abs() * 2.0 ** -8
            for got in (y, z):
                assert bool(((got.double().cpu() - want).abs() <= bound).all())
            assert float((y.double() - z.double()).norm()) <= 0.02 * float(z.double().norm())


def test_example_runs():
    r = example().main(["--steps", "40", "--width", "128", "--heads", "4", "--kv-heads", "2", "--dim", "32", "--lengths", "50", "3", "20", "--chunk", "16", "--singles", "4"])
    assert sum(r["losses"][-5:]) < 0.9 * sum(r["losses"][:5])
    assert r["error"] < 0.1
