"""Rows of long sequences that are formed again pair by pair, because a row that they do not see shares a tile with them and is not finite: that takes
a warp seconds, and no wait of the tensor-core kernels (a second at most) may depend on it.  References: the formulas in 64 bits for single rows."""
import pytest
import torch

import paper_2310_01655_b200 as psk

pytestmark = pytest.mark.gpu
INF = float("inf")


def make(n, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return tuple(torch.randn(1, 1, n, 64, generator=g, device="cuda").bfloat16() for _ in range(4))


def workspace(Q, K, n):
    return torch.empty(psk.binding.window_workspace_bytes(psk.binding.make_window_shape(Q, K, n, 0), True), dtype=torch.uint8, device="cuda")


def weights(Q, K, i):
    """Of row i over the keys 0 .. i."""
    return torch.softmax((K[0, 0, :i + 1].double() @ Q[0, 0, i].double()) * 0.125, 0)


def test_forward():
    n = 1 << 20
    Q, K, V, _ = make(n, 1)
    V[0, 0, 64, 3] = INF                                  # seen by all rows from 64 on
    V[0, 0, n - 2, 7] = INF                               # seen by the last two
    ws = workspace(Q, K, n)
    O, lse = psk.window_attn_fwd(Q, K, V, n, workspace=ws)
    assert psk.check(ws) == 0
    rows = O[0, 0, n - 128:n - 2]
    assert (rows[:, 3] == INF).all() and torch.isfinite(rows[:, [c for c in range(64) if c != 3]]).all()
    assert (O[0, 0, n - 2:, 7] == INF).all() and torch.isfinite(lse).all()
    for i in (n - 128, n - 65, n - 3):
        p, v = weights(Q, K, i), V[0, 0, :i + 1].double()
        v[64, 3] = 0.0
        want, size = p @ v, p @ v.abs()
        # scores in fp32 (2^-15 as for the step), the sum of 2^20 terms in fp32 by 64 lanes' chains (2^-24 a term, of either sign: 2^-12 holds), the output's half step
        off = (O[0, 0, i].double() - want).abs() - (2.0 ** -15 + 2.0 ** -12) * size - 2.0 ** -8 * want.abs()
        assert off[[c for c in range(64) if c != 3]].max() <= 0, i


def test_query_side():
    n = 1 << 19
    Q, K, V, dO = make(n, 2)
    Q[..., 5] = Q[..., 5].abs() + 1
    K[0, 0, 64, 5] = -INF                                 # a weight of nothing in every row from 64 on; 0 times infinity there
    K[0, 0, n - 2, 9] = float("nan")                      # seen by the last two
    ws = workspace(Q, K, n)
    O, lse = psk.window_attn_fwd(Q, K, V, n, workspace=ws)
    assert psk.check(ws) == 0
    dQ = psk.window_attn_bwd(Q, K, V, O, lse, dO, n, workspace=ws)[0]
    assert psk.check(ws) == 0
    keep = [c for c in range(64) if c != 5]
    rows = dQ[0, 0, n - 128:n - 2]
    assert rows[:, 5].isnan().all() and torch.isfinite(rows[:, keep]).all() and dQ[0, 0, n - 2:].isnan().all()
    for i in (n - 128, n - 65, n - 3):
        p, v, k, d = weights(Q, K, i), V[0, 0, :i + 1].double(), K[0, 0, :i + 1].double(), dO[0, 0, i].double()
        k[64] = 0.0
        D, dp = d @ O[0, 0, i].double(), v @ d
        want, size = 0.125 * (p * (dp - D)) @ k, 0.125 * (p * (dp.abs() + D.abs())) @ k.abs()
        off = (dQ[0, 0, i].double() - want).abs() - (2.0 ** -15 + 2.0 ** -12) * size - 2.0 ** -8 * want.abs()
        assert off[keep].max() <= 0, i


def test_key_side():
    n = 1 << 19
    Q, K, V, dO = make(n, 3)
    dO[0, 0, n - 1, 3] = INF                              # seen by all keys: dV is infinite there
    dO[0, 0, 10, 7] = INF                                 # seen by the first eleven
    ws = workspace(Q, K, n)
    O, lse = psk.window_attn_fwd(Q, K, V, n, workspace=ws)
    _, dK, dV = psk.window_attn_bwd(Q, K, V, O, lse, dO, n, workspace=ws)
    assert psk.check(ws) == 0
    keep = [c for c in range(64) if c != 3]
    assert (dV[0, 0, 11:128, 3] == INF).all() and torch.isfinite(dV[0, 0, 11:128][:, keep]).all() and (dV[0, 0, :11, 7] == INF).all()
    for j in (11, 64, 127):
        p = torch.exp((Q[0, 0, j:].double() @ K[0, 0, j].double()) * 0.125 - lse[0, 0, j:].double())
        d = dO[0, 0, j:].double()
        d[-1, 3] = 0.0
        want, size = p @ d, p @ d.abs()
        off = (dV[0, 0, j].double() - want).abs() - (2.0 ** -14 + 2.0 ** -12) * size - 2.0 ** -8 * want.abs()
        assert off[keep].max() <= 0, j
