"""Performance cases of the operators around the attention layer: layer normalisation of its rows, and
sliding-window softmax attention with a cache of fixed size.

What programs do with them:

* "norm": layer normalisation of the rows that attention takes (queries and keys come normalised, rows of one head
  lie inside a projection of queries, keys and values) or of the model's rows; forward alone, or forward and
  backward with the gradients of the gain and the bias;
* "window": softmax attention of every row over the `window` rows up to its own and over the first `sinks` rows of its
  sequence; forward alone with the cache filled behind it (reading a prompt), or forward and backward (training),
  query heads sharing key heads or not, sequences of one batch of different lengths;
* "step": one new token for every sequence of a batch, on that cache.

Shapes are GPT-2's attention layers (12 or 16 heads of 64, model rows of 768 and 1024), from one token of one
sequence to batches of hundreds of thousands of tokens, and odd ones.
"""
import math

import torch

own = False

H_DIM = 64
EPS = 1e-6
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FAR = 2_000_000_000         # positions of a sequence that has been running for a long time


def _norm(dtype, kind, train, n0, n1, n2, cols, **more):
    """kind: "heads" (rows of one head inside a [n0, n2, 3, n1, cols] projection) or "rows" (contiguous)."""
    return dict(more, op="norm", dtype=dtype, kind=kind, train=train, n0=n0, n1=n1, n2=n2, cols=cols)


def _window(dtype, train, B, H, Hkv, n, window, sinks, ragged, **more):
    return dict(more, op="window", dtype=dtype, train=train, B=B, H=H, Hkv=Hkv, n=n, window=window, sinks=sinks, ragged=ragged)


def _step(dtype, B, H, Hkv, window, sinks, mixed, **more):
    """mixed: sequences of all ages in one batch, idle places among them; otherwise all are past their window."""
    return dict(more, op="step", dtype=dtype, B=B, H=H, Hkv=Hkv, window=window, sinks=sinks, mixed=mixed)


def listed():
    return [
        # generating text for one user: the query rows of one token, all latency
        _norm("bf16", "heads", False, 1, 12, 1, 64, name="norm_one_token"),
        # training: the query rows of four sequences of 32k, inside the projection that holds keys and values too
        _norm("bf16", "heads", True, 4, 12, 32768, 64, name="norm_heads_32k"),
        # training: the model's rows in front of a layer, GPT-2 small
        _norm("bf16", "rows", True, 1, 8, 8192, 768, name="norm_model_rows"),
        # fp32 rows of an odd length: no row but the first starts on 16 bytes
        _norm("f32", "rows", True, 1, 5, 777, 1001, name="norm_f32_odd"),
        # generating text for one user: one layer's step for one sequence
        _step("bf16", 1, 12, 12, 1024, 4, False, name="step_one_sequence"),
        # a serving batch with shared key heads and long windows: the caches cross memory once
        _step("bf16", 64, 16, 4, 4096, 4, False, name="step_batch_64"),
        # fp32 caches of sequences of all ages
        _step("f32", 8, 12, 12, 500, 1, True, name="step_f32_mixed"),
        # reading one long prompt of an odd length, and leaving its cache behind
        _window("bf16", False, 1, 12, 12, 16001, 1024, 4, False, name="prompt_16k"),
        # training, GPT-2 small, 131 072 tokens
        _window("bf16", True, 16, 12, 12, 8192, 512, 0, False, name="train_8k_window_512"),
        # a window as long as the sequences: exact causal attention of a short context
        _window("bf16", True, 8, 12, 12, 1024, 1024, 0, False, name="train_1k_causal"),
        # four query heads to a key head, sequences of all lengths from none to the whole, odd sizes
        _window("bf16", True, 5, 16, 4, 1993, 300, 16, True, name="train_shared_ragged"),
        # fp32 training of a small model
        _window("f32", True, 2, 12, 12, 2048, 256, 1, False, name="train_f32_2k"),
    ]


def _log_between(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    op = rng.choice(["norm", "norm", "step", "step", "window", "window", "window"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "norm":
        train = rng.random() < 0.7
        if rng.random() < 0.5:
            H = rng.choice([5, 8, 12, 16, 25])
            n = round(_log_between(rng, 1, 32768))
            B = round(_log_between(rng, 1, max(1.0, 1.5e6 / (n * H))))
            return _norm(dtype, "heads", train, B, H, n, 64)
        cols = round(_log_between(rng, 17, 4096)) if rng.random() < 0.5 else rng.choice([768, 1024, 1280, 2048])
        rows = round(_log_between(rng, 1, 4.0e7 / cols))
        return _norm(dtype, "rows", train, 1, 1, rows, cols)
    Hkv = rng.choice([1, 2, 4, 5, 8, 12])
    H = Hkv * rng.choice([1, 1, 2, 4] if Hkv > 2 else [1, 4, 8])
    if op == "step":
        window, sinks = round(_log_between(rng, 16, 8192)), rng.choice([0, 1, 4, 33])
        most = 5.0e5 if dtype == "bf16" else 2.5e5
        B = round(_log_between(rng, 1, max(1.0, min(128, most / (Hkv * (window + sinks))))))
        return _step(dtype, B, H, Hkv, window, sinks, rng.random() < 0.5)
    train = rng.random() < 0.7
    n = round(_log_between(rng, 1, 8192))
    window = round(_log_between(rng, 1, 2048))
    sinks = rng.choice([0, 0, 1, 4, 70])
    pairs = n * (min(n, window) + 128.0)
    B = round(_log_between(rng, 1, max(1.0, min(24, (4.0e8 if dtype == "bf16" else 6.0e7) / (pairs * H)))))
    return _window(dtype, train, B, H, Hkv, n, window, sinks, rng.random() < 0.4)


# ---- what a program has in hand ----

def _rows_normalised(gen, dtype, *shape):
    x = torch.randn(*shape, generator=gen, device="cuda")
    x = (x - x.mean(-1, keepdim=True)) / (x.var(-1, unbiased=False, keepdim=True) + EPS).sqrt()
    return x.to(DTYPES[dtype])


def _randn(gen, dtype, *shape):
    return torch.randn(*shape, generator=gen, device="cuda").to(DTYPES[dtype])


def _prepare_norm(c, gen):
    n0, n1, n2, cols = c["n0"], c["n1"], c["n2"], c["cols"]
    # rows as a projection leaves them: each with a mean and a spread of its own
    if c["kind"] == "heads":
        X = torch.randn(n0, n2, 3, n1, cols, generator=gen, device="cuda")
        X *= torch.rand(n0, n2, 3, n1, 1, generator=gen, device="cuda") * 2 + 0.25
        X += torch.randn(n0, n2, 3, n1, 1, generator=gen, device="cuda") * 0.5
        X = X.to(DTYPES[c["dtype"]])[:, :, 0].permute(0, 2, 1, 3)
    else:
        X = torch.randn(n0, n1, n2, cols, generator=gen, device="cuda")
        X *= torch.rand(n0, n1, n2, 1, generator=gen, device="cuda") * 2 + 0.25
        X = (X + torch.randn(n0, n1, n2, 1, generator=gen, device="cuda") * 0.5).to(DTYPES[c["dtype"]])
    s = {"c": c, "X": X, "gain": 1 + 0.1 * torch.randn(cols, generator=gen, device="cuda"), "bias": 0.1 * torch.randn(cols, generator=gen, device="cuda")}
    if c["train"]:
        s["dY"] = _randn(gen, c["dtype"], n0, n1, n2, cols)
    return s


def _prepare_window(c, gen):
    B, H, Hkv, n, dt = c["B"], c["H"], c["Hkv"], c["n"], c["dtype"]
    s = {"c": c, "Q": _rows_normalised(gen, dt, B, H, n, H_DIM), "K": _rows_normalised(gen, dt, B, Hkv, n, H_DIM), "V": _randn(gen, dt, B, Hkv, n, H_DIM), "lengths": None}
    if c["ragged"]:
        lengths = (torch.rand(B, generator=gen, device="cuda") * (n + 1)).to(torch.int32).clamp_(max=n)
        # one whole sequence, and where there is room an empty one and one of a single token
        lengths[:3] = torch.tensor([n, 0, 1], dtype=torch.int32, device="cuda")[:min(B, 3)]
        s["lengths"] = lengths
    if c["train"]:
        s["dO"] = _randn(gen, dt, B, H, n, H_DIM)
    else:
        s["Kc"], s["Vc"] = (torch.zeros(B, Hkv, c["sinks"] + c["window"], H_DIM, dtype=DTYPES[dt], device="cuda") for _ in range(2))
    return s


def _prepare_step(c, gen):
    B, H, Hkv, w, dt = c["B"], c["H"], c["Hkv"], c["window"], c["dtype"]
    slots = c["sinks"] + w
    s = {"c": c, "Kc": _rows_normalised(gen, dt, B, Hkv, slots, H_DIM), "Vc": _randn(gen, dt, B, Hkv, slots, H_DIM)}
    s["q"], s["k"], s["v"] = _rows_normalised(gen, dt, B, H, H_DIM), _rows_normalised(gen, dt, B, Hkv, H_DIM), _randn(gen, dt, B, Hkv, H_DIM)
    u = torch.rand(B, generator=gen, device="cuda", dtype=torch.float64)
    pos = slots + (u * 8 * slots).to(torch.int64)
    if c["mixed"]:
        pos = (u * 2 * slots).to(torch.int64)                       # half of them not past their window yet
        pos[:4] = torch.tensor([0, -1, FAR, slots - 1], device="cuda")[:min(B, 4)]
    s["positions"] = pos.to(torch.int32)
    return s


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return {"norm": _prepare_norm, "window": _prepare_window, "step": _prepare_step}[case["op"]](case, gen)


# ---- the framework's calls ----

def _run_own(s):
    import paper_2310_01655_b200 as psk
    c = s["c"]
    if c["op"] == "norm":
        Y = psk.layer_norm_fwd(s["X"], s["gain"], s["bias"], EPS)
        if not c["train"]:
            return {"Y": Y}
        dX, dgain, dbias = psk.layer_norm_bwd(s["X"], s["gain"], s["dY"], EPS)
        return {"Y": Y, "dX": dX, "dgain": dgain, "dbias": dbias}
    if c["op"] == "step":
        o = psk.window_decode_step(s["q"], s["k"], s["v"], s["Kc"], s["Vc"], s["positions"], c["window"], c["sinks"])
        return {"o": o, "Kc": s["Kc"], "Vc": s["Vc"]}
    O, lse = psk.window_attn_fwd(s["Q"], s["K"], s["V"], c["window"], c["sinks"], lengths=s["lengths"])
    if not c["train"]:
        psk.window_cache_fill(s["K"], s["V"], s["Kc"], s["Vc"], c["window"], c["sinks"], lengths=s["lengths"])
        return {"O": O, "lse": lse, "Kc": s["Kc"], "Vc": s["Vc"]}
    dQ, dK, dV = psk.window_attn_bwd(s["Q"], s["K"], s["V"], O, lse, s["dO"], c["window"], c["sinks"], lengths=s["lengths"])
    return {"O": O, "lse": lse, "dQ": dQ, "dK": dK, "dV": dV}


# ---- the plain forms ----

def _plain_norm(s):
    c, gain, bias = s["c"], s["gain"], s["bias"]
    X = s["X"].float()
    X = X - X.mean(-1, keepdim=True)
    rstd = (X.square().mean(-1, keepdim=True) + EPS).rsqrt()
    xhat = X * rstd
    out = {"Y": (xhat * gain + bias).to(s["X"].dtype)}
    if c["train"]:
        dY = s["dY"].float()
        g = dY * gain
        dX = rstd * (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True))
        out["dX"] = dX.to(s["X"].dtype)
        # sums over all rows: a million terms of either sign, in 64 bits
        out["dgain"] = (dY * xhat).sum((0, 1, 2), dtype=torch.float64).float()
        out["dbias"] = dY.sum((0, 1, 2), dtype=torch.float64).float()
    return out


def _blocks(x, nb, size):
    """[.., n, d] -> [.., nb, size, d], zeros behind the end."""
    x = torch.nn.functional.pad(x, (0, 0, 0, nb * size - x.shape[-2]))
    return x.unflatten(-2, (nb, size))


def _with_previous(x):
    """[.., nb, size, d] -> [.., nb, 2 size, d]: the block before (zeros before the first), then the block."""
    prev = torch.nn.functional.pad(x, (0, 0, 0, 0, 1, 0))[..., :-1, :, :]
    return torch.cat([prev, x], -2)


def _sum_of_previous(x):
    """The transpose of _with_previous."""
    prev, mine = x.chunk(2, -2)
    return mine + torch.nn.functional.pad(prev, (0, 0, 0, 0, 0, 1))[..., 1:, :, :]


def _plain_window(s):
    """Blocks of max(window, 64) query rows against their own and the previous block of keys, and against the first
    `sinks` keys where those lie outside the window."""
    c = s["c"]
    B, H, Hkv, n, w, dt = c["B"], c["H"], c["Hkv"], c["n"], c["window"], s["Q"].dtype
    G, scale = H // Hkv, 1 / math.sqrt(H_DIM)
    size = min(max(w, 64), max(n, 1))
    nb = -(-n // size)
    sinks = min(c["sinks"], n)
    dev = s["Q"].device
    lengths = s["lengths"] if s["lengths"] is not None else torch.full((B,), n, dtype=torch.int32, device=dev)
    Q = _blocks(s["Q"].float().view(B, Hkv, G, n, H_DIM), nb, size)                                    # [B,Hkv,G,nb,size,64]
    K, V = (s[x].float() for x in "KV")
    KK, VV = (_with_previous(_blocks(x, nb, size)).unsqueeze(2) for x in (K, V))                       # [B,Hkv,1,nb,2 size,64]
    Ks, Vs = (x[:, :, None, None, :sinks] for x in (K, V))                                             # [B,Hkv,1,1,sinks,64]
    i = torch.arange(nb * size, device=dev).view(nb, size, 1)
    j = torch.arange(-size, size, device=dev).view(1, 1, -1) + torch.arange(0, nb * size, size, device=dev).view(nb, 1, 1)
    js = torch.arange(sinks, device=dev).view(1, 1, -1)
    live = (i < lengths.view(B, 1, 1, 1)).view(B, 1, 1, nb, size, 1)
    band = ((j >= 0) & (j <= i) & (i - j < w)) & live
    early = (js <= i - w) & live
    S = torch.matmul(Q, KK.transpose(-1, -2)).mul_(scale).masked_fill_(~band, -math.inf)
    Ss = torch.matmul(Q, Ks.transpose(-1, -2)).mul_(scale).masked_fill_(~early, -math.inf)
    m = S.amax(-1, keepdim=True)
    m = torch.maximum(m, Ss.amax(-1, keepdim=True)) if sinks else m
    m = m.masked_fill(~live, 0.0)
    S, Ss = S.sub_(m).exp_(), Ss.sub_(m).exp_()
    total = S.sum(-1, keepdim=True) + Ss.sum(-1, keepdim=True)
    over = 1 / total.masked_fill(~live, 1.0)
    P, Ps = S.mul_(over), Ss.mul_(over)
    O = torch.matmul(P, VV) + torch.matmul(Ps, Vs)

    def rows(x):
        return x.flatten(-3, -2)[..., :n, :].reshape(B, H, n, -1)

    out = {"O": rows(O).to(dt), "lse": rows(total.log() + m).squeeze(-1)}
    if not c["train"]:
        # the cache: the first `sinks` positions, then a ring of the last `window` others
        L = lengths.long().view(B, 1)
        slot = torch.arange(c["sinks"] + w, device=dev).view(1, -1)
        r = slot - c["sinks"]
        last = L - 1 - c["sinks"]                                     # the last position, counted from the sinks
        at = torch.where(slot < c["sinks"], slot, c["sinks"] + last - torch.remainder(last - r, w))
        held = torch.where(slot < c["sinks"], slot < L, (last >= 0) & (at >= c["sinks"]))[:, None, :, None]
        take = at.clamp(0, n - 1)[:, None, :, None].expand(B, Hkv, -1, H_DIM)
        for name, x in (("Kc", "K"), ("Vc", "V")):
            s[name].copy_(torch.where(held, s[x].gather(2, take), s[name]))
        return out | {"Kc": s["Kc"], "Vc": s["Vc"]}
    dO = _blocks(s["dO"].float().view(B, Hkv, G, n, H_DIM), nb, size).masked_fill(~live, 0.0)
    D = (dO * O).sum(-1, keepdim=True)
    dV = _sum_of_previous(torch.matmul(P.transpose(-1, -2), dO).sum(2)).flatten(2, 3)[:, :, :n]
    dVs = torch.matmul(Ps.transpose(-1, -2), dO).sum((2, 3))
    dS = torch.matmul(dO, VV.transpose(-1, -2)).sub_(D).mul_(P).mul_(scale)
    dSs = torch.matmul(dO, Vs.transpose(-1, -2)).sub_(D).mul_(Ps).mul_(scale)
    dQ = torch.matmul(dS, KK) + torch.matmul(dSs, Ks)
    dK = _sum_of_previous(torch.matmul(dS.transpose(-1, -2), Q).sum(2)).flatten(2, 3)[:, :, :n]
    dKs = torch.matmul(dSs.transpose(-1, -2), Q).sum((2, 3))
    dK[:, :, :sinks] += dKs
    dV[:, :, :sinks] += dVs
    return out | {"dQ": rows(dQ).to(dt), "dK": dK.to(dt), "dV": dV.to(dt)}


def _plain_step(s):
    c = s["c"]
    B, H, Hkv, w, sinks = c["B"], c["H"], c["Hkv"], c["window"], c["sinks"]
    Kc, Vc, pos = s["Kc"], s["Vc"], s["positions"].long()
    slots = sinks + w
    slot = torch.where(pos < sinks, pos, sinks + torch.remainder(pos - sinks, w))
    mine = (torch.arange(slots, device=pos.device) == slot[:, None]) & (pos >= 0)[:, None]              # [B,slots]
    for cache, x in ((Kc, s["k"]), (Vc, s["v"])):
        cache.copy_(torch.where(mine[:, None, :, None], x[:, :, None], cache))
    held = torch.arange(slots, device=pos.device) <= pos[:, None]                                       # [B,slots]
    q = s["q"].float().view(B, Hkv, H // Hkv, H_DIM)
    S = torch.matmul(q, Kc.float().transpose(-1, -2)) / math.sqrt(H_DIM)
    S = S.masked_fill(~held[:, None, None], -math.inf)
    live = (pos >= 0)[:, None, None, None]
    P = (S - S.amax(-1, keepdim=True).masked_fill(~live, 0.0)).exp()
    P = P / P.sum(-1, keepdim=True).masked_fill(~live, 1.0)
    o = torch.matmul(P, Vc.float()).view(B, H, H_DIM).to(s["q"].dtype)
    return {"o": o, "Kc": Kc, "Vc": Vc}


def run(state):
    if own:
        return _run_own(state)
    return {"norm": _plain_norm, "window": _plain_window, "step": _plain_step}[state["c"]["op"]](state)


def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        rows, cols = case["n0"] * case["n1"] * case["n2"], case["cols"]
        # forward: read X, write Y; backward: read X and dY, write dX; the gain, the bias and their gradients
        n = rows * cols
        return {"bytes": n * size * (5 if case["train"] else 2) + cols * 4 * (5 if case["train"] else 2), "flops": n * (24 if case["train"] else 8)}
    B, H, Hkv, w, sinks = case["B"], case["H"], case["Hkv"], case["window"], case["sinks"]
    if case["op"] == "step":
        # all slots of a sequence past its window; a batch of all ages holds about two thirds of them
        slots = (sinks + w) * (0.66 if case["mixed"] else 1.0)
        return {"bytes": int(2 * B * Hkv * (slots + 2) * H_DIM * size + 2 * B * H * H_DIM * size), "flops": int(4 * B * H * slots * H_DIM)}
    n, share = case["n"], 0.5 if case["ragged"] else 1.0
    inside = min(w, n)
    pairs = inside * (inside + 1) / 2 + (n - inside) * inside + min(sinks, max(0, n - w)) * max(0.0, n - w - sinks / 2)
    q, kv = B * H * n * H_DIM * size, B * Hkv * n * H_DIM * size
    flops = 4 * H_DIM * pairs * B * H * share
    if case["train"]:
        # forward Q, K, V, O; backward Q, K, V, O, dO, dQ, dK, dV; the row statistics written and read
        return {"bytes": int(6 * q + 6 * kv + 8 * B * H * n), "flops": int(3.5 * flops)}
    kept = 2 * B * Hkv * min(n, sinks + w) * H_DIM * size
    return {"bytes": int(2 * q + 2 * kv + 4 * B * H * n + kept), "flops": int(flops)}


# ---- the definitions in 64 bits ----

def _exact_norm(s):
    c = s["c"]
    x, gain, bias = s["X"].double(), s["gain"].double(), s["bias"].double()
    mean = x.mean(-1, keepdim=True)
    std = torch.sqrt((x * x).mean(-1, keepdim=True) - mean * mean + EPS)
    z = (x - mean) / std
    out = {"Y": z * gain + bias}
    if c["train"]:
        d = s["dY"].double()
        dz = d * gain
        out["dX"] = (dz - dz.mean(-1, keepdim=True) - z * (dz * z).mean(-1, keepdim=True)) / std
        out["dgain"] = (d * z).flatten(0, 2).sum(0)
        out["dbias"] = d.flatten(0, 2).sum(0)
    return out


def _exact_window(s):
    """Head by head, the whole matrix of weights."""
    c = s["c"]
    B, H, Hkv, n, w = c["B"], c["H"], c["Hkv"], c["n"], c["window"]
    dev = s["Q"].device
    out = {"O": torch.zeros(B, H, n, H_DIM, dtype=torch.float64, device=dev), "lse": torch.full((B, H, n), -math.inf, dtype=torch.float64, device=dev)}
    if c["train"]:
        out |= {"dQ": torch.zeros_like(out["O"]), "dK": torch.zeros(B, Hkv, n, H_DIM, dtype=torch.float64, device=dev), "dV": torch.zeros(B, Hkv, n, H_DIM, dtype=torch.float64, device=dev)}
    else:
        out |= {"Kc": s["Kc"].double(), "Vc": s["Vc"].double()}
    at = torch.arange(n, device=dev)
    age = at[:, None] - at[None, :]
    sees = (age >= 0) & ((age < w) | (at[None, :] < c["sinks"]))
    lengths = [n] * B if s["lengths"] is None else s["lengths"].tolist()
    for b in range(B):
        L = lengths[b]
        if not c["train"]:
            for p in range(max(0, L - w), L):
                if p >= c["sinks"]:
                    at_slot = c["sinks"] + (p - c["sinks"]) % w
                    out["Kc"][b, :, at_slot], out["Vc"][b, :, at_slot] = s["K"][b, :, p].double(), s["V"][b, :, p].double()
            first = min(c["sinks"], L)
            out["Kc"][b, :, :first], out["Vc"][b, :, :first] = s["K"][b, :, :first].double(), s["V"][b, :, :first].double()
        if L == 0:
            continue
        for h in range(H):
            q, k, v = (s[x][b, y, :L].double() for x, y in (("Q", h), ("K", h // (H // Hkv)), ("V", h // (H // Hkv))))
            a = (q @ k.T / 8.0).masked_fill(~sees[:L, :L], -math.inf)
            lse = torch.logsumexp(a, 1)
            p = torch.exp(a - lse[:, None])
            out["lse"][b, h, :L] = lse
            out["O"][b, h, :L] = p @ v
            if c["train"]:
                g = s["dO"][b, h, :L].double()
                out["dV"][b, h // (H // Hkv), :L] += p.T @ g
                dp = g @ v.T
                da = p * (dp - (p * dp).sum(1, keepdim=True)) / 8.0
                out["dQ"][b, h, :L] = da @ k
                out["dK"][b, h // (H // Hkv), :L] += da.T @ q
    return out


def _exact_step(s):
    c = s["c"]
    B, H, Hkv, w, sinks = c["B"], c["H"], c["Hkv"], c["window"], c["sinks"]
    Kc, Vc = s["Kc"].double(), s["Vc"].double()
    o = torch.zeros(B, H, H_DIM, dtype=torch.float64, device=Kc.device)
    for b, p in enumerate(s["positions"].tolist()):
        if p < 0:
            continue
        slot = p if p < sinks else sinks + (p - sinks) % w
        Kc[b, :, slot], Vc[b, :, slot] = s["k"][b].double(), s["v"][b].double()
        n = min(p + 1, sinks + w)
        k, v = (x[b, :, :n].repeat_interleave(H // Hkv, 0) for x in (Kc, Vc))
        a = torch.softmax(torch.einsum("hd,hnd->hn", s["q"][b].double(), k) / 8.0, -1)
        o[b] = torch.einsum("hn,hnd->hd", a, v)
    return {"o": o, "Kc": Kc, "Vc": Vc}


def exact(case, seed):
    return {"norm": _exact_norm, "window": _exact_window, "step": _exact_step}[case["op"]](prepare(case, seed))
