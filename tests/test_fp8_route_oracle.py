"""The router's oracle where 64 bits hold none of the chosen ones' scores."""
import numpy as np

from oracle import fp8 as ref


def test_oracle_route_of_experts_far_below_the_others():
    """Renormalised weights depend on the chosen logits only: 1000 lower, they are the same, and so are their gradients."""
    bias = np.array([0.0, 2.0, 0.0, 2.0, 2.0])
    x = np.array([[0.5, 1.0, -0.25, 3.0, 2.0]])
    low = x - 1000 * (bias > 0)
    for scale in (1.0, 2.5):
        (w, c), (v, d) = ref.route(x, 3, "softmax", bias, scale=scale), ref.route(low, 3, "softmax", bias, scale=scale)
        assert c.tolist() == [[3, 4, 1]] and d.tolist() == [[1, 3, 4]]      # (lower, all scores are zero: the lowest index first)
        by_hand = np.exp([1.0, 3.0, 2.0]) / np.exp([1.0, 3.0, 2.0]).sum() * scale
        assert np.allclose(v[0], by_hand, rtol=1e-15, atol=0) and np.allclose(w[0], by_hand[[1, 2, 0]], rtol=1e-15, atol=0)
        g = np.array([[0.3, -1.0, 0.7]])
        a, b = ref.route_backward(g, low, d, "softmax", True, scale), ref.route_backward(g[:, [1, 2, 0]], x, c, "softmax", True, scale)
        share = by_hand / scale
        want = np.zeros(5)
        want[[1, 3, 4]] = scale * share * (g[0] - (share * g[0]).sum())
        assert np.allclose(a[0], want, rtol=1e-14, atol=1e-16) and np.allclose(b[0], want, rtol=1e-14, atol=1e-16)
    w, c = ref.route(np.array([[-1000.0, -1001.0, 0.0]]), 2, "sigmoid", [2.0, 2.0, 0.0])
    assert c.tolist() == [[0, 1]] and w.tolist() == [[0.0, 0.0]]
    assert not ref.route_backward(np.ones((1, 2)), np.array([[-1000.0, -1001.0, 0.0]]), c, "sigmoid").any()
