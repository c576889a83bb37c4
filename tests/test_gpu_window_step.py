"""The cache of sliding-window attention and the step of one token on it, and the whole chain of a hybrid layer."""
import numpy as np
import pytest
import torch

import paper_2310_01655_b200 as psk
from paper_2310_01655_b200 import binding
from oracle import window as orc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
# One row: fp32 arithmetic throughout, so a weight is off by ep (68 u times scale sum|q||k|, twice, and 2^-21; with rows of 64
# normal values scale sum|q||k| stays below 16: 1.4e-4 worst case, all of one sign; 2^-15 is what is asked for, the
# square root of the 64 terms of a score being 8 times smaller than their number), plus half a step of the output.
STEP = {"f32": 0.0, "bf16": 2.0 ** -8}
EP = 2.0 ** -15


def f64(x):
    return x.detach().double().cpu().numpy()


def rand(dtype, *shape, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(DT[dtype])


def row(q, K, V, js, scale=0.125):
    s = scale * (K[js] @ q)
    p = np.exp(s - s.max())
    p /= p.sum()
    return p @ V[js], p @ np.abs(V[js])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,window,sinks,steps", [(2, 2, 2, 5, 0, 14), (1, 4, 2, 7, 3, 25), (2, 3, 1, 1, 0, 4), (1, 8, 1, 16, 1, 40), (1, 24, 2, 9, 2, 20),
                                                      (3, 1, 1, 3, 9, 16), (1, 5, 5, 33, 33, 70)])
def test_steps_from_an_empty_cache(dtype, B, H, Hkv, window, sinks, steps):
    q, k, v = rand(dtype, steps, B, H, 64, seed=1), rand(dtype, steps, B, Hkv, 64, seed=2), rand(dtype, steps, B, Hkv, 64, seed=3)
    Kc, Vc = psk.window_cache(B, Hkv, window, sinks, DT[dtype])
    for t in range(steps):
        o = psk.window_decode_step(q[t], k[t], v[t], Kc, Vc, torch.full((B,), t, dtype=torch.int32, device="cuda"), window, sinks)
        js = np.nonzero(orc.visible(t + 1, window, sinks)[t])[0]
        for b in range(B):
            for h in range(H):
                hk = h // (H // Hkv)
                ref, mag = row(f64(q[t, b, h]), f64(k[:, b, hk]), f64(v[:, b, hk]), js)
                assert (np.abs(f64(o[b, h]) - ref) <= EP * mag + STEP[dtype] * np.abs(ref)).all(), (t, b, h)
        for slot, p in orc.cache_slots(window, sinks, t + 1).items():
            assert torch.equal(Kc[:, :, slot], k[p]) and torch.equal(Vc[:, :, slot], v[p])
        assert (Kc[:, :, min(t + 1, sinks + window):] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,H,Hkv,window,sinks", [(1, 1, 1, 255, 0), (1, 12, 12, 1024, 4), (7, 8, 2, 700, 1), (2, 16, 2, 513, 64), (40, 12, 12, 300, 0), (1, 32, 1, 5000, 3),
                                                  (1, 3, 1, 4096, 0), (200, 4, 4, 64, 4)])
def test_mixed_ages(dtype, B, H, Hkv, window, sinks):
    """Sequences at any position, idle places among them: against the slots that are held."""
    slots = window + sinks
    Kc, Vc = rand(dtype, B, Hkv, slots, 64, seed=4), rand(dtype, B, Hkv, slots, 64, seed=5)
    q, k, v = rand(dtype, B, H, 64, seed=6), rand(dtype, B, Hkv, 64, seed=7), rand(dtype, B, Hkv, 64, seed=8)
    g = np.random.default_rng(9)
    pos = np.concatenate([[slots + 5, -1, 0, slots - 1, slots, 2**31 - 1, -2**31, sinks], g.integers(0, 3 * slots, B)])[:B].astype(np.int64)
    # slots that are not held may hold anything
    K1, V1 = Kc.clone(), Vc.clone()
    for b, p in enumerate(pos):
        K1[b, :, max(0, min(p + 1, slots)):] = float("nan")
        V1[b, :, max(0, min(p + 1, slots)):] = float("nan")
    before = K1.clone()
    o = psk.window_decode_step(q, k, v, K1, V1, torch.tensor(pos, dtype=torch.int32, device="cuda"), window, sinks)
    again = psk.window_decode_step(q, k, v, K1, V1, torch.tensor(pos, dtype=torch.int32, device="cuda"), window, sinks)
    assert torch.equal(o, again)
    for b, p in enumerate(pos):
        if p < 0:
            assert (o[b] == 0).all() and torch.equal(K1[b].nan_to_num(9.0), before[b].nan_to_num(9.0))
            continue
        slot = int(p if p < sinks else sinks + (p - sinks) % window)
        assert torch.equal(K1[b, :, slot], k[b]) and torch.equal(V1[b, :, slot], v[b])
        rest = [s for s in range(min(p + 1, slots)) if s != slot]
        assert torch.equal(K1[b][:, rest], Kc[b][:, rest]) and torch.equal(V1[b][:, rest], Vc[b][:, rest])
    for b in sorted({0, B // 2, B - 1} | set(range(min(B, 8)))):
        if pos[b] < 0:
            continue
        js = np.arange(min(pos[b] + 1, slots))
        for h in {0, H // 2, H - 1}:
            hk = h // (H // Hkv)
            ref, mag = row(f64(q[b, h]), f64(K1[b, hk]), f64(V1[b, hk]), js)
            assert (np.abs(f64(o[b, h]) - ref) <= EP * mag + STEP[dtype] * np.abs(ref)).all(), (b, h)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,window,sinks", [(1, 4, 0), (9, 20, 3), (64, 64, 0), (200, 37, 5), (70, 10, 90), (301, 300, 1)])
def test_cache_behind_a_prompt(dtype, n, window, sinks):
    B, Hkv = 5, 3
    proj = rand(dtype, B, n, 2 * Hkv, 64, seed=10)
    K, V = proj[:, :, :Hkv].transpose(1, 2), proj[:, :, Hkv:].transpose(1, 2)
    lens = torch.tensor([n, 0, 1, (n + 1) // 2, n + 7], dtype=torch.int32, device="cuda")
    for lengths in (None, lens):
        Kc, Vc = (torch.full((B, Hkv, sinks + window, 64), 5.0, dtype=DT[dtype], device="cuda") for _ in range(2))
        psk.window_cache_fill(K, V, Kc, Vc, window, sinks, lengths)
        for b in range(B):
            L = n if lengths is None else max(0, min(int(lens[b]), n))
            held = orc.cache_slots(window, sinks, L)
            for slot in range(sinks + window):
                for c, x in ((Kc, K), (Vc, V)):
                    assert torch.equal(c[b, :, slot], x[b, :, held[slot]]) if slot in held else (c[b, :, slot] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_then_tokens(dtype):
    """Normalised rows, a prompt's attention and cache, then tokens one by one: the rows of one long forward."""
    B, H, Hkv, n, more, window, sinks = 3, 4, 2, 150, 40, 60, 4
    total = n + more
    raw = rand(dtype, B, total, H + 2 * Hkv, 64, seed=11)
    gain = 1 + 0.1 * rand("f32", 64, seed=12)
    Q, K, V = (raw[:, :, a:b].transpose(1, 2).contiguous() for a, b in ((0, H), (H, H + Hkv), (H + Hkv, H + 2 * Hkv)))
    Qn, Kn = psk.layer_norm_fwd(Q, gain), psk.layer_norm_fwd(K, gain)
    whole, _ = psk.window_attn_fwd(Qn, Kn, V, window, sinks)
    lens = torch.tensor([n, 17, 0], dtype=torch.int32, device="cuda")
    part = lambda x: x[:, :, :n]
    first, _ = psk.window_attn_fwd(part(Qn), part(Kn), part(V), window, sinks, lengths=lens)
    Kc, Vc = psk.window_cache(B, Hkv, window, sinks, DT[dtype])
    psk.window_cache_fill(part(Kn), part(V), Kc, Vc, window, sinks, lens)
    pos = lens.clone()
    tol = 2.0 ** -14 if dtype == "f32" else 3 * 2.0 ** -8      # (two roundings of the output, one of the weights)
    for b, L in enumerate(lens.tolist()):
        assert np.abs(f64(first[b, :, :L]) - f64(whole[b, :, :L])).max(initial=0) <= 4 * tol
    for t in range(more):
        at = pos.long()[:, None, None, None].expand(B, 1, 1, 64)
        take = lambda x: x.gather(2, at.expand(B, x.shape[1], 1, 64)).squeeze(2)
        # one token's rows, normalised as they come
        q, k = psk.layer_norm_fwd(take(Q), gain), psk.layer_norm_fwd(take(K), gain)
        o = psk.window_decode_step(q, k, take(V), Kc, Vc, pos, window, sinks)
        want = take(whole)
        assert np.abs(f64(o) - f64(want)).max() <= tol * max(1.0, np.abs(f64(want)).max()), t
        pos += 1


def test_hybrid_training_step():
    """Normalised queries and keys into both kinds of attention, the gradients back through the normalisation."""
    B, H, n, window = 1, 2, 256, 64
    X = rand("bf16", 2, B, H, n, 64, seed=13)
    V, d1, d2 = (rand("bf16", B, H, n, 64, seed=s) for s in (14, 15, 16))
    gain = 1 + 0.1 * rand("f32", 64, seed=17)
    g = torch.Generator(device="cuda").manual_seed(18)
    G1, G2 = (torch.randn(H, 64, 16, generator=g, device="cuda").bfloat16() for _ in range(2))
    Q, K = psk.layer_norm_fwd(X[0], gain), psk.layer_norm_fwd(X[1], gain)
    O1, den = psk.causal_attn_fwd(Q, K, V, G1, G2, 128)
    O2, lse = psk.window_attn_fwd(Q, K, V, window, 1)
    a = psk.causal_attn_bwd(Q, K, V, G1, G2, O1, den, d1, 128)
    b = psk.window_attn_bwd(Q, K, V, O2, lse, d2, window, 1)
    gq, gk = (a[i] + b[i] for i in range(2))
    dXq, dgq, dbq = psk.layer_norm_bwd(X[0], gain, gq)
    dXk, dgk, dbk = psk.layer_norm_bwd(X[1], gain, gk)
    rq, rg, rb = orc.layer_norm_backward(f64(X[0]), f64(gain), f64(gq))
    assert np.linalg.norm(f64(dXq) - rq) <= 2 ** -8 * np.linalg.norm(rq) and np.allclose(f64(dgq), rg, rtol=1e-4, atol=1e-4 * np.abs(rg).max())
    for x in (dXk, dgk, dbk, dbq):
        assert torch.isfinite(x).all()
    for h in range(H):
        q, k, v, d = (f64(x[0, h]) for x in (Q, K, V, d2))
        for got, ref in zip(b, orc.window_attention_backward(q, k, v, d, window, 1)):
            assert np.linalg.norm(f64(got[0, h]) - ref) <= 3 * 2 ** -8 * np.linalg.norm(ref)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_graph_stream_and_ctypes(dtype, monkeypatch):
    B, H, Hkv, window, sinks = 3, 8, 2, 400, 2
    Kc, Vc = rand(dtype, B, Hkv, window + sinks, 64, seed=20), rand(dtype, B, Hkv, window + sinks, 64, seed=21)
    q, k, v = rand(dtype, B, H, 64, seed=22), rand(dtype, B, Hkv, 64, seed=23), rand(dtype, B, Hkv, 64, seed=24)
    pos = torch.tensor([5, 401, 9000], dtype=torch.int32, device="cuda")
    copies = lambda: (Kc.clone(), Vc.clone())
    step = lambda c: psk.window_decode_step(q, k, v, *c, pos, window, sinks)
    step(copies())
    c1 = copies()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o1 = step(c1)
        pos.add_(1)
    for _ in range(3):                                  # a captured step advances the positions itself
        graph.replay()
    torch.cuda.synchronize()
    assert pos.tolist() == [8, 404, 9003]
    pos.sub_(3)
    c2 = copies()
    for _ in range(3):
        o2 = step(c2)
        pos.add_(1)
    assert torch.equal(o1, o2) and torch.equal(c1[0], c2[0]) and torch.equal(c1[1], c2[1])
    pos.sub_(1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o3 = step(c2)
    side.synchronize()
    monkeypatch.setattr(binding, "_fast", binding._NoNative())
    o4 = step(c2)
    c5 = copies()
    psk.window_cache_fill(c2[0], c2[1], *c5, window, sinks)
    assert torch.equal(o2, o3) and torch.equal(o2, o4)


def test_refusals():
    Kc, Vc = psk.window_cache(2, 2, 30, 2)
    q, k, v = rand("bf16", 2, 4, 64), rand("bf16", 2, 2, 64), rand("bf16", 2, 2, 64)
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    good = dict(q=q, k=k, v=v, Kc=Kc, Vc=Vc, positions=pos, window=30, sinks=2)
    psk.window_decode_step(**good)
    for bad in (dict(window=31), dict(positions=pos.long()), dict(positions=pos[:1]), dict(k=k[:1]), dict(v=v.float()), dict(Kc=Kc.float()), dict(Kc=Kc[:, :1]),
                dict(q=q.transpose(0, 1)), dict(Vc=Vc.transpose(2, 3).contiguous().transpose(2, 3)), dict(out=q[:, :2]), dict(q=q.half(), k=k.half(), v=v.half())):
        with pytest.raises(ValueError):
            psk.window_decode_step(**(good | bad))
    with pytest.raises(psk.PskError) as e:
        psk.window_decode_step(**(good | dict(scale=-1.0)))
    assert e.value.code == -1
    with pytest.raises(psk.PskError) as e:
        psk.window_decode_step(**(good | dict(q=rand("bf16", 2, 3, 64))))
    assert e.value.code == -3
    with pytest.raises(RuntimeError):
        psk.window_decode_step(**(good | dict(positions=pos.cpu())))
    x = rand("bf16", 2, 2, 9, 64)
    for call in (lambda: psk.window_cache_fill(x, x, Kc, Vc[:1], 30, 2), lambda: psk.window_cache_fill(x, x.float(), Kc, Vc, 30, 2),
                 lambda: psk.window_cache_fill(x, x, Kc, Vc, 29, 2), lambda: psk.window_cache_fill(x, x, Kc, Vc, 30, 2, pos.long())):
        with pytest.raises(ValueError):
            call()


def test_launches_are_counted():
    """What the last call on this thread enqueued, not an earlier one."""
    def launches(call):
        call()
        n = psk.last_launch_count()
        assert n == psk.last_launch_count()
        return n
    Kc, Vc = psk.window_cache(2, 2, 30, 2)
    Q, K, V = rand("bf16", 2, 4, 40, 64, seed=1), rand("bf16", 2, 2, 40, 64, seed=2), rand("bf16", 2, 2, 40, 64, seed=3)
    G = rand("bf16", 1, 64, 16, seed=4)
    X = rand("bf16", 1, 4, 128, 64, seed=5)
    other = launches(lambda: psk.causal_attn_bwd(X, X, X, G, G, X, torch.ones(1, 4, 128, device="cuda"), X, 128))
    assert other > 2
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    O, lse = psk.window_attn_fwd(Q, K, V, 30, 2)
    F = Q.float()
    Kf = K.float()
    Of, lf = psk.window_attn_fwd(F, Kf, Kf, 30)
    for want, call in ((1, lambda: psk.window_attn_fwd(Q, K, V, 30, 2)), (2, lambda: psk.window_attn_bwd(F, F, F, F, torch.zeros(2, 4, 40, device="cuda"), F, 30)),
                       (1, lambda: psk.window_cache_fill(K, V, Kc, Vc, 30, 2)), (1, lambda: psk.window_decode_step(Q[:, :, 0].contiguous(), K[:, :, 0].contiguous(), V[:, :, 0].contiguous(), Kc, Vc, pos, 30, 2)),
                       (1, lambda: psk.layer_norm_fwd(Q)), (1, lambda: psk.layer_norm_bwd(Q, None, Q, params=False)), (2, lambda: psk.layer_norm_bwd(Q, None, Q))):
        assert launches(lambda: psk.causal_attn_bwd(X, X, X, G, G, X, torch.ones(1, 4, 128, device="cuda"), X, 128)) == other
        assert launches(call) == want
    with pytest.raises(psk.PskError):
        psk.window_attn_fwd(Q, K, V, 0)
    assert psk.last_launch_count() == 2                   # (a refused call enqueues nothing and is not counted)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_cache_fill_by_either_binding(dtype, monkeypatch):
    """The native marshalling and ctypes leave the same cache, which is the one that the positions say."""
    B, Hkv, n, window, sinks = 3, 2, 90, 33, 4
    K, V = rand(dtype, B, Hkv, n, 64, seed=51), rand(dtype, B, Hkv, n, 64, seed=52)
    lens = torch.tensor([n, 20, 0], dtype=torch.int32, device="cuda")
    caches = []
    for native in (True, False):
        if not native:
            monkeypatch.setattr(binding, "_fast", binding._NoNative())
        c = tuple(torch.full((B, Hkv, sinks + window, 64), 3.0, dtype=DT[dtype], device="cuda") for _ in range(2))
        psk.window_cache_fill(K, V, *c, window, sinks, lens)
        caches.append(c)
    for a, b, x in zip(*caches, (K, V)):
        assert torch.equal(a, b)
        for i, L in enumerate(lens.tolist()):
            held = orc.cache_slots(window, sinks, L)
            for slot in range(sinks + window):
                assert torch.equal(a[i, :, slot], x[i, :, held[slot]]) if slot in held else (a[i, :, slot] == 3).all()
