"""fp64 CPU definitions of layer normalisation and sliding-window softmax attention, with their gradients.

Written from the formulas, pair by pair where it matters; shares no code with the CUDA library.  Arrays of one head: Q, K,
V, dO [n, h]; rows from `length` on are behind the sequence's end."""
import numpy as np


def layer_norm(X, gain=None, bias=None, eps=1e-6):
    X = np.asarray(X, dtype=np.float64)
    mean = X.mean(axis=-1, keepdims=True)
    var = ((X - mean) ** 2).mean(axis=-1, keepdims=True)
    Y = (X - mean) / np.sqrt(var + eps)
    if gain is not None:
        Y = Y * gain
    return Y if bias is None else Y + bias


def layer_norm_backward(X, gain, dY, eps=1e-6):
    """(dX, dgain, dbias), the last two summed over all rows."""
    X, dY = np.asarray(X, dtype=np.float64), np.asarray(dY, dtype=np.float64)
    mean = X.mean(axis=-1, keepdims=True)
    rstd = 1 / np.sqrt(((X - mean) ** 2).mean(axis=-1, keepdims=True) + eps)
    xhat = (X - mean) * rstd
    a = dY if gain is None else dY * gain
    dX = rstd * (a - a.mean(axis=-1, keepdims=True) - xhat * (a * xhat).mean(axis=-1, keepdims=True))
    rows = tuple(range(X.ndim - 1))
    return dX, (dY * xhat).sum(axis=rows), dY.sum(axis=rows)


def visible(n, window, sinks, length=None):
    """[n, n] truth values: does row i see row j?"""
    length = n if length is None else max(0, min(length, n))
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    return (i < length) & (j <= i) & ((i - j < window) | (j < sinks))


def window_attention(Q, K, V, window, sinks=0, scale=None, length=None):
    """(O, lse, P): pairs that the mask leaves out are never formed, so what stands in their rows does not matter."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    n, h = Q.shape
    scale = h ** -0.5 if scale is None else scale
    M = visible(n, window, sinks, length)
    O, lse, P = np.zeros((n, h)), np.full(n, -np.inf), np.zeros((n, n))
    for i in range(n):
        js = np.nonzero(M[i])[0]
        if len(js) == 0:
            continue
        s = scale * (K[js] @ Q[i])
        m = s.max()
        e = np.exp(s - m)
        lse[i] = m + np.log(e.sum())
        P[i, js] = e / e.sum()
        O[i] = (e / e.sum()) @ V[js]
    return O, lse, P


def window_attention_backward(Q, K, V, dO, window, sinks=0, scale=None, length=None):
    """(dQ, dK, dV) of one query head."""
    Q, K, V, dO = (np.asarray(x, dtype=np.float64) for x in (Q, K, V, dO))
    n, h = Q.shape
    scale = h ** -0.5 if scale is None else scale
    M = visible(n, window, sinks, length)
    O, _, P = window_attention(Q, K, V, window, sinks, scale, length)
    dQ, dK, dV = np.zeros((n, h)), np.zeros((n, h)), np.zeros((n, h))
    for i in range(n):
        js = np.nonzero(M[i])[0]
        if len(js) == 0:
            continue
        p = P[i, js]
        ds = p * (V[js] @ dO[i] - dO[i] @ O[i]) * scale
        dQ[i] = ds @ K[js]
        dK[js] += np.outer(ds, Q[i])
        dV[js] += np.outer(p, dO[i])
    return dQ, dK, dV


def cache_slots(window, sinks, length):
    """{slot: position} that the cache holds behind `length` positions."""
    held = {}
    for p in range(length):
        held[p if p < sinks else sinks + (p - sinks) % window] = p
    return held
