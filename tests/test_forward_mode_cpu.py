"""Forward-mode derivatives of what is differentiable, without a GPU: the launch is replaced by torch operations."""
import pytest

torch = pytest.importorskip("torch")

import torch.autograd.forward_ad as forward_ad  # noqa: E402

from paper_1912_12607_amd import positions  # noqa: E402


def _plain(x, at, frequencies, back):
    t = at.double()[..., None, None] * frequencies * (-1.0 if back else 1.0)
    n = frequencies.numel()
    a, b = x[..., :n], x[..., n:2 * n]
    return torch.cat([a * t.cos() - b * t.sin(), a * t.sin() + b * t.cos(), x[..., 2 * n:]], -1)


@pytest.fixture
def rotary(monkeypatch):
    """A Rotary whose launches are torch operations on what the tensors hold (as a kernel, they see no tangent)."""
    r = positions.Rotary(6)

    def turn(plan, q, k, at, back):
        with torch.no_grad():
            out = tuple(torch.empty_like(x).copy_(_plain(forward_ad.unpack_dual(x).primal.detach(), at, r.frequencies, back)) for x in (q, k) if x is not None)
        return out
    monkeypatch.setattr(r, "_check", lambda q, k, at: (q.shape, None if k is None else k.shape))
    monkeypatch.setattr(r, "_turn", turn)
    monkeypatch.setattr(r, "_launch", lambda *a: None)
    return r


AT = torch.tensor([0, 3, 1000], dtype=torch.int32)


def normal(*shape, seed=0):
    return torch.randn(*shape, dtype=torch.float64, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("grad", [True, False])
def test_tangents_are_turned_as_what_they_belong_to(rotary, grad):
    q, k, tq, tk = normal(3, 4, 8), normal(3, 2, 8, seed=1), normal(3, 4, 8, seed=2), normal(3, 2, 8, seed=3)

    def near(a, b):
        assert torch.allclose(a, b, rtol=0, atol=1e-12)
    with forward_ad.dual_level(), torch.set_grad_enabled(grad):
        y = forward_ad.unpack_dual(rotary(forward_ad.make_dual(q, tq), None, AT))
        near(y.primal, _plain(q, AT, rotary.frequencies, 0)), near(y.tangent, _plain(tq, AT, rotary.frequencies, 0))
        for dq, dk in ((1, 1), (1, 0), (0, 1)):
            out = rotary(forward_ad.make_dual(q, tq) if dq else q, forward_ad.make_dual(k, tk) if dk else k, AT)
            for o, x, t, has in zip(out, (q, k), (tq, tk), (dq, dk)):
                near(forward_ad.unpack_dual(o).primal, _plain(x, AT, rotary.frequencies, 0))
                near(forward_ad.unpack_dual(o).tangent, _plain(t, AT, rotary.frequencies, 0) if has else torch.zeros_like(x))
        assert forward_ad.unpack_dual(rotary(q, k, AT)[0]).tangent is None


def test_tangents_of_gradients(rotary):
    """Forward over reverse: the gradient of sum(y^2) / 2 at q is q itself (turns keep lengths), its tangent q's tangent."""
    q, t = normal(3, 4, 8).requires_grad_(True), normal(3, 4, 8, seed=2)
    for k in (None, normal(3, 2, 8, seed=1)):
        with forward_ad.dual_level():
            x = forward_ad.make_dual(q, t)
            y = rotary(x, k, AT)
            y = y if k is None else y[0]
            d, = torch.autograd.grad((y * y).sum() / 2, x)
            d = forward_ad.unpack_dual(d)
            assert torch.allclose(d.primal, q, rtol=0, atol=1e-12) and torch.allclose(d.tangent, t, rtol=0, atol=1e-12)


def test_gradients_of_tangents(rotary):
    q, t, g = normal(3, 4, 8), normal(3, 4, 8, seed=2).requires_grad_(True), normal(3, 4, 8, seed=3)
    with forward_ad.dual_level():
        d, = torch.autograd.grad(forward_ad.unpack_dual(rotary(forward_ad.make_dual(q, t), None, AT)).tangent, t, g)
    assert torch.allclose(d, _plain(g, AT, rotary.frequencies, 1), rtol=0, atol=1e-12)


def test_in_place_takes_no_tangents(rotary):
    q = normal(3, 4, 8)
    with forward_ad.dual_level():
        with pytest.raises(RuntimeError, match="gradients"):
            rotary.turn_(forward_ad.make_dual(q, q.clone()), None, AT)
        with pytest.raises(RuntimeError, match="gradients"):
            rotary.turn_(q, forward_ad.make_dual(q.clone(), q.clone()), AT)
        rotary.turn_(q, None, AT)
