"""Forward-mode derivatives on the GPU: a tangent is turned by the same kernel, so that it equals the turn of the tangent alone."""
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

import torch.autograd.forward_ad as forward_ad  # noqa: E402

from paper_1912_12607_amd import fourbit, tokens  # noqa: E402
from paper_1912_12607_amd.positions import Rotary  # noqa: E402

DEV = torch.device("cuda:0")


def normal(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_rotary(dtype, layout):
    rotary, at = Rotary(10, layout=layout, amplitude=1.5), torch.tensor([0, 3, 100000], dtype=torch.int32, device=DEV)
    q, k, tq, tk = (normal(3, h, 16, seed=i, dtype=dtype) for i, h in enumerate((4, 2, 4, 2)))
    plain, turned = rotary(q, k, at), rotary(tq, tk, at)
    with forward_ad.dual_level():
        for grad in (True, False):
            with torch.set_grad_enabled(grad):
                for dq, dk in ((1, 1), (1, 0), (0, 1)):
                    out = rotary(forward_ad.make_dual(q, tq) if dq else q, forward_ad.make_dual(k, tk) if dk else k, at)
                    for o, p, t, has in zip(out, plain, turned, (dq, dk)):
                        o = forward_ad.unpack_dual(o)
                        assert torch.equal(o.primal, p) and torch.equal(o.tangent, t if has else torch.zeros_like(t))
                assert torch.equal(forward_ad.unpack_dual(rotary(forward_ad.make_dual(q, tq), None, at)).tangent, turned[0])
        with pytest.raises(RuntimeError, match="gradients"):
            rotary.turn_(forward_ad.make_dual(q.clone(), tq), None, at)
        # forward over reverse: the tangent of a gradient is turned back
        x, g = q.clone().requires_grad_(True), normal(3, 4, 16, seed=7, dtype=dtype)
        d, = torch.autograd.grad(rotary(x, k, at)[0], x, forward_ad.make_dual(g, tq))
        d = forward_ad.unpack_dual(d)
    for gradient, got in ((g, d.primal), (tq, d.tangent)):
        assert torch.equal(got, torch.autograd.grad(rotary(x, None, at), x, gradient)[0])


def test_transformations_are_refused():
    rotary, at, q = Rotary(16), torch.zeros(3, dtype=torch.int32, device=DEV), normal(3, 4, 16)
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda x: rotary(x, None, at), (q,), (q,))
    with pytest.raises(RuntimeError):
        torch.func.vmap(lambda x: rotary(x, None, at))(q.expand(2, 3, 4, 16))


@pytest.mark.parametrize("layer", [tokens.linear, fourbit.linear4])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_linear_layers_refuse_tangents(layer, which):
    """Of their arguments, and of the gradient that comes in (forward over reverse): none is dropped."""
    args = [normal(5, 64), normal(32, 64, seed=1), normal(32, seed=2)]
    with forward_ad.dual_level():
        for grad in (True, False):
            with torch.set_grad_enabled(grad), pytest.raises(RuntimeError):
                layer(*(forward_ad.make_dual(a, a.clone()) if i == which else a for i, a in enumerate(args)))
        leaves = [a.clone().requires_grad_(i == which) for i, a in enumerate(args)]
        y = layer(*leaves)
        g = normal(5, 32, seed=3)
        with pytest.raises(RuntimeError, match="forward mode"):
            torch.autograd.grad(y, leaves[which], forward_ad.make_dual(g, g.clone()))
        assert torch.isfinite(torch.autograd.grad(layer(*leaves), leaves[which], g)[0]).all()
