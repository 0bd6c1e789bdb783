"""Pins of the fp64 oracle of the operators on rows: finite differences, autograd and closed forms."""
import numpy as np
import pytest
import torch

from oracle import qk_rmsnorm_numpy as per_head
from oracle import row_ops_numpy as orn


def _draw(seed, *shape):
    return np.random.default_rng(seed).standard_normal(shape)


@pytest.mark.parametrize("scale", [True, False])
@pytest.mark.parametrize("D", [1, 2, 7, 40])
def test_tangents_are_directional_derivatives(D, scale):
    x, res, tx, tres = (_draw(k, 5, D) for k in range(4))
    g = 1 + 0.3 * _draw(9, D) if scale else None
    step, eps = 1e-5, 1e-3

    def y(sign):
        return orn.rmsnorm_jvp_fwd(x + sign * step * tx, res + sign * step * tres, None, None, g, eps)["y"][0]

    out = orn.rmsnorm_jvp_fwd(x, res, tx, tres, g, eps)
    assert np.allclose(out["ty"][0], (y(1) - y(-1)) / (2 * step), rtol=1e-7, atol=1e-8)
    assert np.array_equal(out["h"][0], x + res) and np.array_equal(out["th"][0], tx + tres)


@pytest.mark.parametrize("tangent", [True, False])
@pytest.mark.parametrize("D", [1, 3, 24])
def test_backward_is_the_gradient_of_the_forward(D, tangent):
    """Against torch's autograd through the forward written with a jvp."""
    x, res, tx, tres, dy, dty, dh, dth = (torch.from_numpy(_draw(k, 4, D)) for k in range(8))
    g = torch.from_numpy(1 + 0.3 * _draw(9, D))
    leaves = [t.requires_grad_() for t in (x, res, tx, tres, g)]
    eps = 1e-3
    h, t = x + res, tx + tres

    def norm(v):
        return v / (v.square().mean(-1, keepdim=True) + eps).sqrt()

    u, jt = torch.autograd.functional.jvp(norm, h, t, create_graph=True)
    loss = (dy * g * u).sum() + (dh * h).sum()
    if tangent:
        loss = loss + (dty * g * jt).sum() + (dth * t).sum()
    dx, dres, dtx, dtres, dg = torch.autograd.grad(loss, leaves, allow_unused=True)
    n = [v.detach().numpy() for v in (h, dy, t, dty, dh, dth, g)]
    out = orn.rmsnorm_jvp_bwd(n[0], n[1], n[2] if tangent else None, n[3], n[4], n[5], n[6], eps)
    assert np.allclose(out["dx"][0], dx.numpy(), rtol=1e-9, atol=1e-11) and torch.equal(dx, dres)
    assert np.allclose(out["dg"][0], dg.numpy(), rtol=1e-9, atol=1e-11)
    if tangent:
        assert np.allclose(out["dtx"][0], dtx.numpy(), rtol=1e-9, atol=1e-11) and torch.equal(dtx, dtres)
    else:
        assert out["dtx"][0] is None


def test_agrees_with_the_per_head_oracle():
    x, tx, dy, dty = (_draw(k, 2, 3, 5, 16) for k in range(4))
    g = 1 + 0.3 * _draw(9, 16)
    out = orn.rmsnorm_jvp_fwd(x, None, tx, None, g, 1e-6)
    y, ty = per_head.rmsnorm_jvp_fwd(x, tx, g, 1e-6)
    assert np.allclose(out["y"][0], y) and np.allclose(out["ty"][0], ty)
    back = orn.rmsnorm_jvp_bwd(x, dy, tx, dty, None, None, g, 1e-6)
    for got, want in zip((back["dx"][0], back["dtx"][0], back["dg"][0]), per_head.rmsnorm_jvp_bwd(x, tx, g, dy, dty, 1e-6)):
        assert np.allclose(got, want, rtol=1e-10, atol=1e-12)


def test_sizes_bound_the_values():
    x, tx, dy, dty = (_draw(k, 6, 10) for k in range(4))
    for out in (orn.rmsnorm_jvp_fwd(x, None, tx, None, None, 1e-6), orn.rmsnorm_jvp_bwd(x, dy, tx, dty, None, None, None, 1e-6)):
        for value, size in out.values():
            assert (np.abs(value) <= size * (1 + 1e-12)).all()


def test_rows_in_8_bits_and_products_of_small_cases():
    s, v = orn.rows_to_8_bits(np.array([[254.0, -127.0, 1.0], [0.0, 0.0, 0.0]]))
    assert np.array_equal(s, [2.0, 0.0]) and np.array_equal(v, [[127.0, -63.5, 0.5], [0.0, 0.0, 0.0]])
    q, w = np.array([[127, -128]], np.int8), np.array([[-128, 127], [1, 1]], np.int8)
    y, size = orn.linear_s8(q, np.array([0.5]), w, np.array([1.0, 2.0]), np.array([1.0, -1.0]))
    assert np.array_equal(y, [[0.5 * (-127 * 128 - 128 * 127) + 1, 0.5 * 2 * -1 - 1]]) and np.array_equal(size, [[0.5 * 2 * 127 * 128 + 1, 2.0]])
