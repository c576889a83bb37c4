"""Sliding-window attention, forward and backward, against the definition in 64 bits, element by element.

Tolerances, from the roundings that the kernels make (u = 2^-24; e = 2^-8, half a step of bf16, or u for fp32 storage):
* a score is off by (64 + 4) u scale sum|q||k| at most, so is its row's lse; with the exponential's 2^-22 a weight p is off by
  p ep, ep = 2 * 68 u scale max_j sum|q||k_j| + 2^-21;
* o = sum p v: p is rounded once as an operand (e, fp32: not), the sum over N rows in fp32 adds N u of its terms: error
  (ep + e + N u) sum p|v|, plus the output's own rounding;
* D = do.o from the stored o: |do|.(error of o) + 64 u |do|.|o|; do.v: 64 u |do|.|v|;
* ds = p (do.v - D): |ds| (ep + e) + p (both errors); dq, dk, dv sum these times |k|, |q|, and (ep + e + N u) p times |do|."""
import numpy as np
import pytest
import torch

import paper_2310_01655_b200 as psk
from paper_2310_01655_b200 import binding
from oracle import window as orc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
E = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
U = 2.0 ** -24


def f64(x):
    return x.detach().double().cpu().numpy()


def make(dtype, B, H, Hkv, n, seed=0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda h: torch.randn(B, h, n, 64, generator=g, device="cuda")
    return tuple(x.to(DT[dtype]) for x in (r(H) * spread, r(Hkv) * spread, r(Hkv), r(H)))


def within(name, got, ref, tol):
    got = f64(got)
    assert np.array_equal(np.isfinite(got), np.isfinite(ref)), name
    fine = np.isfinite(ref)
    # (a weight below 2^-126, fp32's smallest normal number, becomes 0: an error of at most 2^-126 for each, and a result is a sum of
    # fewer than 2^16 of them times factors below 2^10)
    off = np.abs(np.where(fine, got, 0) - np.where(fine, ref, 0))[fine] - np.broadcast_to(tol, ref.shape)[fine] - 2.0 ** -100
    assert off.size == 0 or off.max() <= 0, "%s: off by %.3e more than allowed (%.3e)" % (name, off.max(), np.broadcast_to(tol, ref.shape)[fine].max())


def check_heads(dtype, Q, K, V, dO, out, window, sinks, scale=None, lengths=None, heads=None):
    """out: (O, lse, dQ, dK, dV) or (O, lse); whole groups of query heads that share a key head are looked at."""
    B, H, n, _ = Q.shape
    Hkv, G = K.shape[1], H // K.shape[1]
    sc = 0.125 if scale is None else scale
    e = E[dtype]
    p_e = e if dtype == "bf16" else 0.0
    for b, hk in (heads or {(0, 0), (B - 1, Hkv - 1)}):
        L = None if lengths is None else int(lengths[b])
        k, v = f64(K[b, hk]), f64(V[b, hk])
        dk, dv, tk, tv = (np.zeros((n, 64)) for _ in range(4))
        for h in range(hk * G, hk * G + G):
            q = f64(Q[b, h])
            M = orc.visible(n, window, sinks, L)
            k0, v0, q0 = (np.where(np.isfinite(x), x, 0) for x in (k, v, q))
            O, lse, P = orc.window_attention(q, k, v, window, sinks, sc, L)
            S = np.where(M, np.abs(q0) @ np.abs(k0).T, 0) * sc
            ep = 2 * 68 * U * S.max(1, keepdims=True) + 2.0 ** -21
            N = M.sum(1, keepdims=True) + 64
            t_o = (ep + p_e + N * U) * (P @ np.abs(v0)) + e * np.abs(O)
            within("O[%d,%d]" % (b, h), out[0][b, h], O, t_o)
            within("lse[%d,%d]" % (b, h), out[1][b, h], lse, (ep[:, 0] + N[:, 0] * U) + 4 * U * np.abs(np.where(np.isfinite(lse), lse, 0)))
            if len(out) == 2:
                continue
            d = f64(dO[b, h])
            d0 = np.where(np.isfinite(d), d, 0)
            rq, rk, rv = orc.window_attention_backward(q, k, v, d, window, sinks, sc, L)
            D = (d0 * O).sum(1, keepdims=True)
            dp = np.where(M, d0 @ v0.T, 0)
            eD = (np.abs(d0) * t_o).sum(1, keepdims=True) + 64 * U * (np.abs(d0) * np.abs(O)).sum(1, keepdims=True)
            eds = np.abs(P * (dp - D)) * (ep + p_e + 4 * U) + P * (eD + 64 * U * np.where(M, np.abs(d0) @ np.abs(v0).T, 0))
            N2 = (M.sum(0)[:, None] * G + 64) * U
            ds = np.abs(P * (dp - D)) + eds
            within("dQ[%d,%d]" % (b, h), out[2][b, h], rq, sc * (eds + N * U * ds) @ np.abs(k0) + (e + 2 * U) * np.abs(rq))
            dk += rk
            dv += rv
            tk += sc * (eds.T @ np.abs(q0) + N2 * (ds.T @ np.abs(q0)))
            tv += (P * (ep + p_e)).T @ np.abs(d0) + N2 * (P.T @ np.abs(d0))
        if len(out) > 2:
            within("dK[%d,%d]" % (b, hk), out[3][b, hk], dk, tk + (e + 2 * U) * (np.abs(dk) + tk))
            within("dV[%d,%d]" % (b, hk), out[4][b, hk], dv, tv + (e + 2 * U) * (np.abs(dv) + tv))


def run(Q, K, V, dO, window, sinks=0, **more):
    ws = torch.empty(psk.binding.window_workspace_bytes(psk.binding.make_window_shape(Q, K, window, sinks), True), dtype=torch.uint8, device="cuda")
    O, lse = psk.window_attn_fwd(Q, K, V, window, sinks, workspace=ws, **more)
    assert psk.check(ws) == 0
    grads = psk.window_attn_bwd(Q, K, V, O, lse, dO, window, sinks, workspace=ws, **more)
    assert psk.check(ws) == 0
    return (O, lse) + grads


PATHS = [("f32", psk.PATH_AUTO), ("bf16", psk.PATH_AUTO), ("bf16", psk.PATH_CUDA_CORES)]


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("B,H,Hkv,n,window,sinks", [
    (1, 1, 1, 1, 1, 0), (1, 1, 1, 1, 50, 3), (1, 2, 1, 2, 1, 0), (2, 2, 2, 5, 2, 1), (1, 1, 1, 63, 17, 0), (1, 1, 1, 64, 64, 0), (1, 3, 1, 65, 33, 2),
    (2, 2, 2, 127, 200, 0), (1, 2, 2, 128, 128, 0), (1, 1, 1, 129, 1, 0), (1, 4, 2, 200, 1, 5), (1, 2, 2, 255, 63, 0), (1, 1, 1, 256, 64, 64),
    (1, 1, 1, 257, 65, 1), (1, 2, 1, 300, 100, 130), (2, 4, 4, 320, 129, 4), (1, 8, 1, 385, 96, 7), (1, 1, 1, 385, 2**31 - 1, 0),
    (1, 1, 1, 300, 20, 2**31 - 1), (1, 1, 1, 513, 127, 3), (1, 2, 2, 640, 128, 0), (1, 6, 2, 700, 260, 200), (1, 1, 1, 897, 256, 16)])
def test_against_the_definition(dtype, path, B, H, Hkv, n, window, sinks):
    Q, K, V, dO = make(dtype, B, H, Hkv, n, seed=n + window % 1000)
    out = run(Q, K, V, dO, window, sinks, path=path)
    check_heads(dtype, Q, K, V, dO, out, window, sinks)
    for x, y in zip(out, run(Q, K, V, dO, window, sinks, path=path)):
        assert torch.equal(x, y)                              # every sum in a fixed order


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("window,sinks", [(40, 0), (150, 5), (300, 140), (1000, 0)])
def test_sequences_of_all_lengths(dtype, path, window, sinks):
    n = 391
    lengths = [n, 0, 1, 63, 64, 65, 127, 128, 129, 200, 256, 257, 390, -5, n + 9]
    Q, K, V, dO = make(dtype, len(lengths), 2, 1, n, seed=window)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = run(Q, K, V, dO, window, sinks, path=path, lengths=lens)
    for b, L in enumerate(lengths):
        L = max(0, min(L, n))
        assert (out[0][b, :, L:] == 0).all() and (out[1][b, :, L:] == float("-inf")).all()
        assert all((x[b, :, L:] == 0).all() for x in out[2:])
    check_heads(dtype, Q, K, V, dO, out, window, sinks, lengths=lens.tolist(), heads=[(b, 0) for b in range(len(lengths))])
    # what stands behind a sequence's end does not count
    for b, L in enumerate(lengths):
        L = max(0, min(L, n))
        for x in (Q, K, V, dO):
            x[b, :, L:] = float("nan") if b % 2 else float("inf")
    for x, y in zip(out, run(Q, K, V, dO, window, sinks, path=path, lengths=lens)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("B,H,Hkv,n,window,sinks,lengths", [
    (1, 1, 1, 1400, 40, 4, None), (2, 4, 2, 1111, 100, 64, [1111, 300]), (1, 2, 1, 1500, 1, 1, None), (3, 2, 2, 900, 64, 100, [0, 150, 900]),
    (2, 3, 1, 2050, 129, 128, [2049, 2050]), (1, 2, 2, 700, 30, 200, None), (4, 1, 1, 1000, 65, 2, [1, 2, 320, 321])])
def test_sinks_of_long_sequences(dtype, path, B, H, Hkv, n, window, sinks, lengths):
    """The sinks are seen by every row: their gradients may be added up from several parts."""
    Q, K, V, dO = make(dtype, B, H, Hkv, n, seed=n)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = run(Q, K, V, dO, window, sinks, path=path, lengths=lens)
    check_heads(dtype, Q, K, V, dO, out, window, sinks, lengths=lengths, heads=[(b, Hkv - 1) for b in range(B)])
    for b in range(B if lengths else 0):
        assert all(x[b, :, lengths[b]:].eq(0).all() for x in out[2:])
    for x, y in zip(out, run(Q, K, V, dO, window, sinks, path=path, lengths=lens)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("row", [10, 700])
def test_sinks_of_long_sequences_with_infinities(dtype, path, row):
    """A row of dO that is infinite in one column, among the rows of the sinks' tile or of a part: the sinks' gradients are what the sums say."""
    Q, K, V, dO = make(dtype, 1, 2, 1, 1200, seed=3)
    dO[0, 1, row, 5] = float("inf")
    out = run(Q, K, V, dO, 50, 3, path=path)
    check_heads(dtype, Q, K, V, dO, out, 50, 3)


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("window,sinks", [(70, 0), (200, 3), (2000, 0)])
def test_masked_infinities_and_nans(dtype, path, bad, window, sinks):
    """A row is not touched by what stands in rows that it does not see, not even where both lie in one tile."""
    n = 450
    Q, K, V, dO = make(dtype, 1, 2, 1, n, seed=17)
    for s in (201, 330):
        later, earlier = slice(s, None), slice(None, s)
        Q2, K2, V2, d2 = (x.clone() for x in (Q, K, V, dO))
        for x in (Q2, K2, V2, d2):
            x[:, :, later] = bad
        got = run(Q2, K2, V2, d2, window, sinks, path=path)
        part = lambda x: x[:, :, earlier].contiguous()
        assert torch.isfinite(got[0][:, :, earlier]).all() and torch.isfinite(got[2][:, :, earlier]).all()
        check_heads(dtype, part(Q), part(K), part(V), part(dO), (part(got[0]), part(got[1])), window, sinks)
        rq = orc.window_attention_backward(f64(Q[0, 1])[:s], f64(K[0, 0])[:s], f64(V[0, 0])[:s], f64(dO[0, 1])[:s], window, sinks)[0]
        assert np.linalg.norm(f64(got[2][0, 1, earlier]) - rq) <= 4 * max(E[dtype], 1e-6) * np.linalg.norm(rq)
        # keys behind the last bad query row: of earlier queries nothing counts
        Q2, d2 = Q.clone(), dO.clone()
        for x in (Q2, d2):
            x[:, :, earlier] = bad
        got = run(Q2, K, V, d2, window, sinks, path=path)
        clean = run(Q, K, V, dO, window, sinks, path=path)
        for x, y, name in zip(got[3:], clean[3:], ("dK", "dV")):
            x, y = f64(x[:, :, later]), f64(y[:, :, later])
            assert np.isfinite(x).all(), name
            assert np.linalg.norm(x - y) <= 4 * max(E[dtype], 1e-6) * np.linalg.norm(y), name
    # and a key too old to be seen
    if window < n:
        K2, V2 = K.clone(), V.clone()
        K2[:, :, 100] = bad
        V2[:, :, 100] = bad
        got = run(Q, K2, V2, dO, window, sinks, path=path)
        assert torch.isfinite(got[0][:, :, 100 + window:]).all() and torch.isfinite(got[2][:, :, 100 + window:]).all()
        assert not torch.isfinite(got[0][:, :, 100:100 + window].float()).any(-1).any()


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("B,H,Hkv,n,window,sinks,lengths", [
    (1, 8, 1, 700, 300, 0, None), (2, 12, 2, 333, 333, 0, [333, 100]), (1, 16, 1, 1500, 200, 3, None), (3, 6, 1, 600, 500, 70, [0, 599, 65]),
    (1, 10, 2, 513, 2000, 1, [512]), (1, 3, 1, 1111, 600, 0, None), (1, 32, 1, 150, 100, 0, None)])
def test_few_key_heads(dtype, path, B, H, Hkv, n, window, sinks, lengths):
    """Many query heads to few key heads: their gradients may be added up from several groups of heads."""
    Q, K, V, dO = make(dtype, B, H, Hkv, n, seed=n + H)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = run(Q, K, V, dO, window, sinks, path=path, lengths=lens)
    check_heads(dtype, Q, K, V, dO, out, window, sinks, lengths=lengths, heads=[(b, Hkv - 1) for b in range(B)])
    for b in range(B if lengths else 0):
        assert all(x[b, :, lengths[b]:].eq(0).all() for x in out[2:])
    for x, y in zip(out, run(Q, K, V, dO, window, sinks, path=path, lengths=lens)):
        assert torch.equal(x, y)
    # keys inside a projection: what lies between them is left as it was
    both = torch.full((2, B, n, Hkv, 2, 64), 3.0, dtype=DT[dtype], device="cuda")
    dK, dV = (both[i, :, :, :, i].transpose(1, 2) for i in range(2))
    K2 = torch.zeros_like(both[0])
    Ks, Vs = K2[:, :, :, 0].transpose(1, 2), K2[:, :, :, 1].transpose(1, 2)
    Ks.copy_(K), Vs.copy_(V)
    psk.window_attn_bwd(Q, Ks, Vs, out[0], out[1], dO, window, sinks, lengths=lens, path=path, out=(torch.empty_like(Q), dK, dV))
    assert torch.equal(dK, out[3]) and torch.equal(dV, out[4])
    assert (both[0, :, :, :, 1] == 3).all() and (both[1, :, :, :, 0] == 3).all()


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("window,sinks", [(200, 0), (150, 40), (2000, 0)])
def test_few_key_heads_with_infinities(dtype, path, bad, window, sinks):
    n, s = 700, 333
    Q, K, V, dO = make(dtype, 1, 8, 1, n, seed=41)
    Q[0, 5, s] = bad                       # one query row of one of the eight heads
    got = run(Q, K, V, dO, window, sinks, path=path)
    clean = make(dtype, 1, 8, 1, n, seed=41)
    good = run(clean[0], K, V, dO, window, sinks, path=path)
    seen = torch.zeros(n, dtype=torch.bool, device="cuda")
    seen[max(0, s - window + 1):s + 1] = True
    seen[:min(sinks, s + 1)] = True
    for x, y in zip(got[3:], good[3:]):
        assert not torch.isfinite(x[0, 0, seen].float()).any() and torch.isfinite(x[0, 0, ~seen].float()).all()
        a, b = x[0, 0, ~seen].double(), y[0, 0, ~seen].double()
        assert (a - b).norm() <= 4 * max(E[dtype], 1e-6) * b.norm()


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("which", ["q row", "k row", "k", "v", "dO", "all"])
@pytest.mark.parametrize("window,sinks", [(70, 0), (60, 130), (2000, 0)])
def test_infinities_and_nans_that_are_seen(dtype, path, bad, which, window, sinks):
    """What is not finite by the formulas, and only that, comes out so; all else is as if alone."""
    n, s = 420, 131
    Q, K, V, dO = make(dtype, 1, 2, 1, n, seed=29)
    if which == "q row":
        Q[0, 1, s] = bad
    elif which == "k row":
        K[0, 0, s] = bad
    elif which == "k":
        K[0, 0, s, 9] = bad
    elif which == "v":
        V[0, 0, s, 9] = bad
    elif which == "dO":
        dO[0, 1, s, 9] = bad
    else:
        for x in (Q, K, V, dO):
            x.fill_(bad)
    got = run(Q, K, V, dO, window, sinks, path=path)
    with np.errstate(all="ignore"):
        dk = dv = 0.0
        pairs = []
        for h in range(2):
            a = (f64(Q[0, h]), f64(K[0, 0]), f64(V[0, 0]))
            O, lse, _ = orc.window_attention(*a, window, sinks, 0.125)
            rq, rk, rv = orc.window_attention_backward(*a, f64(dO[0, h]), window, sinks, 0.125)
            pairs += [("O", got[0][0, h], O), ("lse", got[1][0, h], lse), ("dQ", got[2][0, h], rq)]
            dk, dv = dk + rk, dv + rv
        pairs += [("dK", got[3][0, 0], dk), ("dV", got[4][0, 0], dv)]
        for name, x, y in pairs:
            x = f64(x)
            fine = np.isfinite(y)
            assert np.array_equal(np.isfinite(x), fine), name
            assert np.linalg.norm((x - y)[fine]) <= 4 * max(E[dtype], 1e-6) * np.linalg.norm(y[fine]), name


@pytest.mark.parametrize("dtype,path", PATHS)
def test_large_scores(dtype, path):
    # weights that are one or nothing, scores in the hundreds, growing along the row so that the running maximum moves on
    n, window = 300, 170
    Q, K, V, dO = make(dtype, 1, 1, 1, n, seed=3, spread=4.0)
    K = (K.float() * torch.linspace(0.2, 3.0, n, device="cuda")[None, None, :, None]).to(K.dtype)
    out = run(Q, K, V, dO, window, 2, path=path)
    check_heads(dtype, Q, K, V, dO, out, window, 2)
    out = run(Q, K.flip(2).contiguous(), V, dO, window, 2, path=path)
    check_heads(dtype, Q, K.flip(2), V, dO, out, window, 2)


@pytest.mark.parametrize("dtype,path", PATHS)
@pytest.mark.parametrize("scale", [1e-4, 0.3, 1.0])
def test_scales(dtype, path, scale):
    Q, K, V, dO = make(dtype, 1, 2, 2, 150, seed=4)
    out = run(Q, K, V, dO, 70, 1, path=path, scale=scale)
    check_heads(dtype, Q, K, V, dO, out, 70, 1, scale=scale)


@pytest.mark.parametrize("dtype,path", PATHS)
def test_inside_a_projection(dtype, path):
    """[B, n, (H + 2 Hkv), 64] as a projection leaves it; queries and keys have strides of their own."""
    B, n, H, Hkv, window, sinks = 2, 333, 4, 2, 90, 3
    g = torch.Generator(device="cuda").manual_seed(6)
    proj = torch.randn(B, n, H + 2 * Hkv, 64, generator=g, device="cuda").to(DT[dtype])
    Q, K, V = (proj[:, :, a:b].transpose(1, 2) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    dO = torch.empty_strided(Q.shape, Q.stride(), dtype=Q.dtype, device="cuda")
    dO.copy_(torch.randn(B, H, n, 64, generator=g, device="cuda"))
    before = proj.clone()
    out = run(Q, K, V, dO, window, sinks, path=path)
    assert torch.equal(proj, before) and out[0].stride() == Q.stride() and out[3].stride() == K.stride()
    dense = run(*(x.contiguous() for x in (Q, K, V, dO)), window, sinks, path=path)
    for x, y in zip(out, dense):
        assert torch.equal(x, y)
    # outputs into a buffer of gradients of the projection: what lies between is left as it was
    gp = torch.full_like(proj, 7.0)
    views = tuple(gp[:, :, a:b].transpose(1, 2) for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    psk.window_attn_bwd(Q, K, V, out[0], out[1], dO, window, sinks, path=path, out=views)
    for x, y in zip(views, out[2:]):
        assert torch.equal(x, y)
    with pytest.raises(ValueError):
        psk.window_attn_bwd(Q, K, V, out[0].contiguous(), out[1], dO, window, sinks, path=path)


@pytest.mark.parametrize("dtype,path", PATHS)
def test_rows_far_apart(dtype, path):
    # element offsets that pass 32 bits
    n, step = 140, 17_000_000
    Q, K, V, dO = make(dtype, 1, 1, 1, n, seed=7)
    big = torch.empty(n * step, dtype=Q.dtype, device="cuda")
    far = lambda x, at: big.as_strided((1, 1, n, 64), (n * step, n * step, step, 1), at).copy_(x)
    ref = run(Q, K, V, dO, 50, 2, path=path)
    q, k, v, d = (far(x, 64 * i) for i, x in enumerate((Q, K, V, dO)))
    outs = [big.as_strided((1, 1, n, 64), (n * step, n * step, step, 1), 64 * (4 + i)) for i in range(4)]
    O, lse = psk.window_attn_fwd(q, k, v, 50, 2, path=path, out=outs[0])
    grads = psk.window_attn_bwd(q, k, v, O, lse, d, 50, 2, path=path, out=tuple(outs[1:]))
    for x, y in zip((O, lse) + tuple(grads), ref):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_stream_and_ctypes(dtype, monkeypatch):
    Q, K, V, dO = make(dtype, 2, 4, 2, 270, seed=8)
    lens = torch.tensor([270, 111], dtype=torch.int32, device="cuda")

    def step():
        O, lse = psk.window_attn_fwd(Q, K, V, 100, 3, lengths=lens)
        return (O, lse) + psk.window_attn_bwd(Q, K, V, O, lse, dO, 100, 3, lengths=lens)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for x, y in zip((Q, K, V, dO), make(dtype, 2, 4, 2, 270, seed=9)):
        x.copy_(y)
    lens.copy_(torch.tensor([33, 270]))
    graph.replay()
    torch.cuda.synchronize()
    ref = step()
    for x, y in zip(got, ref):
        assert torch.equal(x, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    side.synchronize()
    monkeypatch.setattr(binding, "_fast", binding._NoNative())
    for x, y, z in zip(ref, other, step()):
        assert torch.equal(x, y) and torch.equal(x, z)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_streams_at_once(dtype):
    sets = [make(dtype, 2, 3, 3, 600, seed=30 + i) for i in range(2)]
    refs = [run(*s, 130, 2) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    outs = [[], []]
    for _ in range(5):
        for i, (st, s) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(st):
                O, lse = psk.window_attn_fwd(*s[:3], 130, 2)
                outs[i].append((O, lse) + psk.window_attn_bwd(*s[:3], O, lse, s[3], 130, 2))
    torch.cuda.synchronize()
    for ref, got in zip(refs, outs):
        for one in got:
            for x, y in zip(ref, one):
                assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_are_differences(dtype):
    """Along random directions: d/de sum(O . dO), O from the oracle's forward (64 bits) at the stored inputs."""
    n, window, sinks = 90, 30, 2
    Q, K, V, dO = make(dtype, 1, 1, 1, n, seed=10)
    grads = run(Q, K, V, dO, window, sinks)[2:]
    q, k, v, d = (f64(x[0, 0]) for x in (Q, K, V, dO))
    g = np.random.default_rng(11)
    f = lambda *a: (orc.window_attention(*a, window, sinks)[0] * d).sum()
    for i, got in enumerate(grads):
        D = f64(got[0, 0]) + np.linalg.norm(f64(got[0, 0])) / 80 * g.normal(size=(n, 64))       # (a direction that the gradient is not small along)
        a = lambda s: f(*[x + s * 1e-5 * D if j == i else x for j, x in enumerate((q, k, v))])
        diff = (a(1) - a(-1)) / 2e-5
        # errors of the gradient's elements are at most 3 half steps (p or ds, the output, D) and of either sign
        assert abs(diff - (f64(got[0, 0]) * D).sum()) <= 3 * max(E[dtype], 1e-6) * np.linalg.norm(f64(got[0, 0])) * np.linalg.norm(D)


def test_refusals():
    Q, K, V, dO = make("bf16", 2, 4, 2, 40)
    lens = torch.tensor([40, 3], dtype=torch.int32, device="cuda")
    O, lse = psk.window_attn_fwd(Q, K, V, 8)
    for call in (lambda: psk.window_attn_fwd(Q, K, V[:, :, :39], 8), lambda: psk.window_attn_fwd(Q, K.float(), V.float(), 8),
                 lambda: psk.window_attn_fwd(Q.half(), K.half(), V.half(), 8), lambda: psk.window_attn_fwd(Q, K, V, 8, lengths=lens.long()),
                 lambda: psk.window_attn_fwd(Q, K, V, 8, lengths=lens[:1]), lambda: psk.window_attn_fwd(Q, K[:1], V[:1], 8),
                 lambda: psk.window_attn_fwd(Q[0], K, V, 8), lambda: psk.window_attn_fwd(Q, K, V, 8, lse=lse.double()),
                 lambda: psk.window_attn_fwd(Q, K, V, 8, out=O.float()), lambda: psk.window_attn_fwd(Q, K, V, 8, workspace=lse),
                 lambda: psk.window_attn_bwd(Q, K, V, O, lse[:1], dO, 8), lambda: psk.window_attn_bwd(Q, K, V, O, lse, dO.float(), 8)):
        with pytest.raises(ValueError):
            call()
    for call, code in ((lambda: psk.window_attn_fwd(Q, K, V, 0), -3), (lambda: psk.window_attn_fwd(Q, K, V, 8, -1), -3),
                       (lambda: psk.window_attn_fwd(Q, K, V, 8, scale=0.0), -1), (lambda: psk.window_attn_fwd(Q[:, :3].contiguous(), K, V, 8), -3),
                       (lambda: psk.window_attn_fwd(Q[..., :32].contiguous(), K[..., :32].contiguous(), V[..., :32].contiguous(), 8), -2),
                       (lambda: psk.window_attn_fwd(Q.float(), K.float(), V.float(), 8, path=psk.PATH_TENSOR_CORES), -2),
                       (lambda: psk.window_attn_fwd(Q[:, :1].expand(2, 4, 40, 64), K, V, 8), -3),
                       (lambda: psk.window_attn_fwd(Q, K, V, 8, workspace=torch.empty(8, dtype=torch.uint8, device="cuda")), -5)):
        with pytest.raises(psk.PskError) as e:
            call()
        assert e.value.code == code
    with pytest.raises(RuntimeError):
        psk.window_attn_fwd(Q, K.cpu(), V.cpu(), 8)


def test_windows_beyond_32_bits():
    Q, K, V, dO = make("bf16", 1, 2, 1, 40)
    O, lse = psk.window_attn_fwd(Q, K, V, 2**31 - 1, 2**31 - 1)
    q, k, v = Q[:, :, 0], K[:, :, 0], V[:, :, 0]
    Kc, Vc = psk.window_cache(1, 1, 8)
    pos = torch.zeros(1, dtype=torch.int32, device="cuda")
    for window, sinks in ((2**32 + 8, 0), (8, 2**32), (2**31, 0)):
        for call in (lambda: psk.window_attn_fwd(Q, K, V, window, sinks), lambda: psk.window_attn_bwd(Q, K, V, O, lse, dO, window, sinks)):
            with pytest.raises(psk.PskError) as e:
                call()
            assert e.value.code == -3
        for call in (lambda: psk.window_decode_step(q, k, v, Kc, Vc, pos, window, sinks), lambda: psk.window_cache_fill(K, V, Kc, Vc, window, sinks)):
            with pytest.raises((psk.PskError, ValueError)):
                call()


@pytest.mark.parametrize("B,H,Hkv,n,window,sinks,lengths", [
    (1, 2, 2, 200, 1, 0, None), (1, 2, 1, 200, 2, 0, None), (2, 2, 2, 333, 3, 1, [333, 70]), (1, 4, 2, 300, 8, 0, None), (1, 2, 2, 260, 40, 2, None), (1, 1, 1, 400, 400, 0, None),
    (30, 8, 4, 150, 2, 0, None)])
def test_the_rounding_of_the_stored_output_does_not_reach_the_gradients(B, H, Hkv, n, window, sinks, lengths):
    """bf16 on the tensor cores.  D0 = do . o from the stored o is off by R = D - D0, |R| <= |do| . (o's error); with few keys to a row that is as large as
    ds itself.  The kernels take it out again, R being the sum of the row's p (dP - D0), off by
    eR = (ep + (N + 8) u) sum p |dP - D0| + 64 u sum p |do||v|.  Then dQ sums ds' = p (dP - D0) and p, each rounded once (e), the latter times R; dK sums ds
    formed with D0 + R: errors |ds| (ep + e) + p |R| 2 e + p eR (+ 64 u p |do||v| and the sums' N u), times |k|; without p |R| 2 e times |q|."""
    Q, K, V, dO = make("bf16", B, H, Hkv, n, seed=n + window)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    O, lse, dQ, dK, dV = run(Q, K, V, dO, window, sinks, lengths=lens)
    e, G = E["bf16"], H // Hkv
    for b, hk in {(0, 0), (B - 1, Hkv - 1)}:
        k, v = f64(K[b, hk]), f64(V[b, hk])
        dk, tk = np.zeros((n, 64)), np.zeros((n, 64))
        for h in range(hk * G, hk * G + G):
            q, d, L = f64(Q[b, h]), f64(dO[b, h]), None if lengths is None else lengths[b]
            M = orc.visible(n, window, sinks, L)
            o, _, P = orc.window_attention(q, k, v, window, sinks, 0.125, L)
            rq, rk, _ = orc.window_attention_backward(q, k, v, d, window, sinks, 0.125, L)
            N = M.sum(1, keepdims=True) + 64
            ep = 2 * 68 * U * np.where(M, np.abs(q) @ np.abs(k).T, 0).max(1, keepdims=True) * 0.125 + 2.0 ** -21
            dp, D, dv = np.where(M, d @ v.T, 0), (d * o).sum(1, keepdims=True), np.where(M, np.abs(d) @ np.abs(v).T, 0)
            R = (np.abs(d) * ((ep + e + N * U) * (P @ np.abs(v)) + e * np.abs(o))).sum(1, keepdims=True) + 64 * U * (np.abs(d) * np.abs(o)).sum(1, keepdims=True)
            ds = np.abs(P * (dp - D))
            eR = (ep + (N + 8) * U) * (ds + P * R).sum(1, keepdims=True) + 64 * U * (P * dv).sum(1, keepdims=True)
            both = ds * (ep + e + 4 * U) + P * (eR + 64 * U * dv + 4 * U * np.abs(D))
            eq = both + P * R * (2 * e + ep)
            within("dQ[%d,%d]" % (b, h), dQ[b, h], rq, 0.125 * (eq + N * U * (ds + P * R + eq)) @ np.abs(k) + (e + 2 * U) * np.abs(rq))
            dk += rk
            tk += 0.125 * (both.T @ np.abs(q) + (M.sum(0)[:, None] * G + 64) * U * ((ds + both).T @ np.abs(q)))
        within("dK[%d,%d]" % (b, hk), dK[b, hk], dk, tk + (e + 2 * U) * (np.abs(dk) + tk))
