"""Pins of the attention block's gradients in the oracle: against central
differences of its forward, and the plain layer's backward where the weights
cannot change."""
import numpy as np

import workloads
from oracle import attention, layer

NAMES = ("x", "W", "edge_vec", "radial_w", "W1", "w2")


def _problem(seed, L=2, C=8, R=6, H=2, F=5, N=7, E=40):
    w = workloads.random_graph(seed, n_nodes=N, n_edges=E, L=L, C=C, R=R)
    rng = np.random.default_rng(seed)
    d = (L + 1) ** 2
    fac = [rng.standard_normal((d, R)) / np.sqrt(d) for _ in range(3)]
    W1 = 2 * rng.standard_normal((2 * C + w["n_radial"], F)) / np.sqrt(2 * C)
    w2 = rng.standard_normal((F, H))
    return w, fac, W1, w2


def test_gradients_match_differences():
    w, (A, B, D), W1, w2 = _problem(3)
    val = dict(x=w["x"], W=w["W"], edge_vec=w["edge_vec"], radial_w=w["radial_w"], W1=W1, w2=w2)
    val = {k: np.asarray(v, np.float64) for k, v in val.items()}

    def loss(v):
        out, _ = attention.forward(v["x"], w["edge_index"], v["edge_vec"], A, B, D, v["W"], v["radial_w"], v["W1"],
                                   v["w2"], w["r_cut"], 2)
        return (out * w["grad_out"]).sum()

    grads = attention.backward(val["x"], w["edge_index"], val["edge_vec"], A, B, D, val["W"], val["radial_w"], W1, w2,
                               w["r_cut"], 2, w["grad_out"])
    probe = np.random.default_rng(4)
    for name, g in zip(NAMES, grads):
        assert g.shape == val[name].shape
        for _ in range(3):
            u = probe.standard_normal(g.shape)
            step = 1e-6
            diff = (loss({**val, name: val[name] + step * u}) - loss({**val, name: val[name] - step * u})) / (2 * step)
            assert abs((g * u).sum() - diff) < 2e-6 * (1 + abs(diff)), name


def test_single_edges_have_the_layers_gradients():
    # one edge into each of four nodes: alpha = 1 whatever the logits
    w, (A, B, D), W1, w2 = _problem(5, N=8, E=4)
    w["edge_index"] = np.array([[0, 1, 2, 0], [4, 5, 6, 7]], np.int32)
    args = (w["x"], w["edge_index"], w["edge_vec"], A, B, D, w["W"], w["radial_w"])
    gx, gW, gv, gr, g1, g2 = attention.backward(*args, W1, w2, w["r_cut"], 2, w["grad_out"])
    ref = layer.backward(*args, w["r_cut"], 2, w["grad_out"], return_radial=True)
    for a, b in zip((gx, gW, gv, gr), ref):
        np.testing.assert_allclose(a, b, rtol=1e-11, atol=1e-12)
    assert np.abs(g1).max() < 1e-12 and np.abs(g2).max() < 1e-12


def test_the_absolute_chain_bounds_every_gradient():
    w, (A, B, D), W1, w2 = _problem(6)
    args = (w["x"], w["edge_index"], w["edge_vec"], A, B, D, w["W"], w["radial_w"], W1, w2, w["r_cut"], 2,
            w["grad_out"])
    for g, s in zip(attention.backward(*args), attention.backward(*args, absolute=True)):
        assert np.all(np.abs(g) <= s * (1 + 1e-12) + 1e-300)
