"""The fp64 definitions of layer normalisation and sliding-window attention, checked against themselves: differences,
torch's own autograd in 64 bits, and the cache's slots against the mask."""
import numpy as np
import pytest
import torch

from oracle import window as orc


def central(f, x, d, step=1e-6):
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("rows,cols", [((3,), 5), ((2, 4), 64), ((1,), 1)])
def test_layer_norm_gradients_are_differences(rows, cols):
    g = np.random.default_rng(cols)
    X, dY = g.normal(size=rows + (cols,)), g.normal(size=rows + (cols,))
    gain, bias = g.normal(size=cols), g.normal(size=cols)
    dX, dgain, dbias = orc.layer_norm_backward(X, gain, dY)
    D, e = g.normal(size=X.shape), g.normal(size=cols)
    # (one column: y does not depend on x)
    assert np.isclose(central(lambda x: (orc.layer_norm(x, gain, bias) * dY).sum(), X, D), (dX * D).sum(), rtol=1e-6, atol=1e-7)
    assert np.isclose(central(lambda x: (orc.layer_norm(X, x, bias) * dY).sum(), gain, e), (dgain * e).sum(), rtol=1e-7, atol=1e-8)
    assert np.isclose(central(lambda x: (orc.layer_norm(X, gain, x) * dY).sum(), bias, e), (dbias * e).sum(), rtol=1e-7, atol=1e-8)


@pytest.mark.parametrize("n,window,sinks,length", [(7, 3, 0, None), (9, 2, 3, None), (9, 100, 0, 6), (6, 1, 0, None), (5, 2, 9, 0), (8, 3, 1, 1)])
def test_window_gradients_are_differences_and_autograd(n, window, sinks, length):
    g = np.random.default_rng(n + window)
    h = 4
    Q, K, V, dO = (g.normal(size=(n, h)) for _ in range(4))
    O, lse, _ = orc.window_attention(Q, K, V, window, sinks, 0.7, length)
    grads = orc.window_attention_backward(Q, K, V, dO, window, sinks, 0.7, length)
    for k in range(3):
        D = g.normal(size=(n, h))
        args = lambda x: [x if i == k else y for i, y in enumerate((Q, K, V))]
        diff = central(lambda x: (orc.window_attention(*args(x), window, sinks, 0.7, length)[0] * dO).sum(), (Q, K, V)[k], D)
        assert np.isclose(diff, (grads[k] * D).sum(), rtol=1e-6, atol=1e-8)
    t = [torch.tensor(x, requires_grad=True) for x in (Q, K, V)]
    M = torch.tensor(orc.visible(n, window, sinks, length))
    s = (t[0] @ t[1].T * 0.7).masked_fill(~M, -1e300)
    out = (torch.softmax(s, 1) * M) @ t[2]
    assert np.allclose(out.detach().numpy(), O, atol=1e-12)
    out.backward(torch.tensor(dO))
    for x, ref in zip(t, grads):
        assert np.allclose(x.grad.numpy(), ref, atol=1e-12)
    assert np.array_equal(np.isinf(lse), ~orc.visible(n, window, sinks, length).any(1))


def test_pairs_that_do_not_count_bring_nothing_in():
    g = np.random.default_rng(3)
    n, w, s, L = 12, 3, 2, 9
    Q, K, V, dO = (g.normal(size=(n, 4)) for _ in range(4))
    clean = orc.window_attention(Q, K, V, w, s, None, L)[:2] + orc.window_attention_backward(Q, K, V, dO, w, s, None, L)
    for x in (Q, K, V, dO):
        x[L:] = np.nan
    again = orc.window_attention(Q, K, V, w, s, None, L)[:2] + orc.window_attention_backward(Q, K, V, dO, w, s, None, L)
    for x, y in zip(clean, again):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 0), (3, 2), (5, 1), (2, 7)])
def test_the_cache_holds_what_the_next_row_sees(window, sinks):
    for t in range(25):
        held = orc.cache_slots(window, sinks, t + 1)
        assert sorted(held) == list(range(min(t + 1, sinks + window)))          # the slots below, and all of them
        assert sorted(held.values()) == list(np.nonzero(orc.visible(t + 1, window, sinks)[t])[0])
