"""Pins of the oracle of the norm and the feed-forward block: the token case
against torch's own, rotations commute, gradients against differences."""
import numpy as np
import pytest
import torch

from oracle import block, sh

EPS = 1e-5


def _norm_inputs(seed, N, L, C):
    rng = np.random.default_rng(seed)
    d = (L + 1) ** 2
    return (rng.standard_normal((N, d, C)) + 0.3, 1 + 0.2 * rng.standard_normal((L + 1, C)),
            0.2 * rng.standard_normal(C), rng.standard_normal((N, d, C)))


def _ffn_inputs(seed, N, L, C, F):
    rng = np.random.default_rng(seed)
    d = (L + 1) ** 2
    return (rng.standard_normal((N, d, C)), rng.standard_normal((C, F)) / C ** 0.5,
            rng.standard_normal((C, F)) / C ** 0.5, rng.standard_normal((F, C)) / F ** 0.5,
            0.3 * rng.standard_normal(F), rng.standard_normal((N, d, C)))


def test_layer_norm_of_scalars_is_torchs():
    x, g, b, dy = _norm_inputs(1, 7, 0, 16)
    t = torch.from_numpy(x[:, 0]).requires_grad_()
    gt, bt = torch.from_numpy(g[0]).requires_grad_(), torch.from_numpy(b).requires_grad_()
    y = torch.nn.functional.layer_norm(t, (16,), gt, bt, EPS)
    np.testing.assert_allclose(block.layer_norm(x, g, b, EPS)[:, 0], y.detach().numpy(), rtol=1e-12, atol=1e-13)
    y.backward(torch.from_numpy(dy[:, 0]))
    gx, gg, gb = block.layer_norm_backward(x, g, dy, EPS)
    np.testing.assert_allclose(gx[:, 0], t.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(gg[0], gt.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(gb, bt.grad.numpy(), rtol=1e-12)


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_activations_are_torchs(act):
    q = np.linspace(-9, 9, 301)
    t = torch.from_numpy(q).requires_grad_()
    y = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "sigmoid": torch.sigmoid}[act](t)
    y.sum().backward()
    a, da = block.activation(q, act)
    np.testing.assert_allclose(a, y.detach().numpy(), rtol=1e-12, atol=1e-15)
    np.testing.assert_allclose(da, t.grad.numpy(), rtol=1e-10, atol=1e-14)


def _differences(f, v, probe, step=1e-6):
    """Central differences of f along random directions of v."""
    for _ in range(3):
        u = probe.standard_normal(v.shape)
        yield u, (f(v + step * u) - f(v - step * u)) / (2 * step)


@pytest.mark.parametrize("L", [0, 2])
def test_layer_norm_gradients_match_differences(L):
    x, g, b, dy = _norm_inputs(2, 5, L, 16)
    probe = np.random.default_rng(5)
    grads = block.layer_norm_backward(x, g, dy, EPS)
    for k, (v, grad) in enumerate(zip((x, g, b), grads)):
        def f(t, k=k):
            a = [x, g, b]
            a[k] = t
            return (block.layer_norm(*a, EPS) * dy).sum()
        for u, diff in _differences(f, v, probe):
            assert abs((grad * u).sum() - diff) < 1e-6 * (1 + abs(diff))


@pytest.mark.parametrize("act", ["silu", "gelu", "sigmoid"])
def test_gated_ffn_gradients_match_differences(act):
    x, wu, wg, wd, b, dy = _ffn_inputs(3, 4, 1, 16, 32)
    probe = np.random.default_rng(6)
    args = [x, wu, wg, wd, b]
    grads = block.gated_ffn_backward(x, wu, wg, wd, dy, b, act)
    for k, (v, grad) in enumerate(zip(args, grads)):
        def f(t, k=k):
            a = list(args)
            a[k] = t
            return (block.gated_ffn(*a, act=act) * dy).sum()
        for u, diff in _differences(f, v, probe):
            assert abs((grad * u).sum() - diff) < 1e-6 * (1 + abs(diff))


def test_both_commute_with_rotations():
    L, C, F, N = 3, 16, 32, 4
    d = (L + 1) ** 2
    rng = np.random.default_rng(8)
    q, r = np.linalg.qr(rng.standard_normal((3, 3)))
    rot = q * np.sign(np.diag(r))
    if np.linalg.det(rot) < 0:
        rot[:, 0] *= -1
    # the representation from harmonics at sample directions: Y(R v) = D Y(v)
    v = rng.standard_normal((200, 3))
    big = np.linalg.lstsq(sh.spherical_harmonics(L, v), sh.spherical_harmonics(L, v @ rot.T), rcond=None)[0].T
    x, g, b, _ = _norm_inputs(9, N, L, C)
    turn = lambda t: np.einsum("ij,njc->nic", big, t)  # noqa: E731
    np.testing.assert_allclose(block.layer_norm(turn(x), g, b, EPS), turn(block.layer_norm(x, g, b, EPS)), atol=1e-9)
    _, wu, wg, wd, bg, _ = _ffn_inputs(10, N, L, C, F)
    np.testing.assert_allclose(block.gated_ffn(turn(x), wu, wg, wd, bg), turn(block.gated_ffn(x, wu, wg, wd, bg)),
                               atol=1e-9)
    assert d == big.shape[0]
