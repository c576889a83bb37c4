"""Layer normalisation, forward and backward, against the definition in 64 bits.

Tolerances (u = 2^-24, C columns, one row; sums are trees of at most t = C / 32 + 12 additions deep in a lane):
* xhat: the mean is off by at most t u max|x|, a deviation by that and its own rounding, rstd by (t + 4) u relative, so that with
  A = max|x| rstd every entry is within (2 t + 8) u (A + |xhat|) of the exact one; y adds two roundings, and half a step of the
  storage type (bf16: 2^-8 |y|, fp32: in the rounding already counted);
* dx = rstd (a - m1 - xhat m2): with S = rstd (max|a| + max|xhat| max|a xhat|) the two means are off by t u of their
  largest terms and xhat by the above: (4 t + 24) u S (1 + A) covers them, plus the storage type's half step;
* dgain, dbias: n rows summed in chunks: relative to the sum of the terms' magnitudes (64 + (2 t + 8) (1 + A)) u."""
import numpy as np
import pytest
import torch

import paper_2310_01655_b200 as psk
from paper_2310_01655_b200 import binding
from oracle import window as orc

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
U = 2.0 ** -24
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def f64(x):
    return x.detach().double().cpu().numpy()


def rows_of(dtype, *shape, seed=0, offset=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(*shape, generator=g, device="cuda")
    x = x * (torch.rand(*shape[:-1], 1, generator=g, device="cuda") * 2 + 0.25) + offset * torch.randn(*shape[:-1], 1, generator=g, device="cuda")
    return x.to(DT[dtype])


def within(name, got, ref, tol):
    got = f64(got)
    off = np.abs(got - ref) - tol
    assert np.isfinite(got).all() and off.max() <= 0, "%s: off by %.3e more than allowed (%.3e)" % (name, off.max(), np.asarray(tol).max())


def check(dtype, X, gain, bias, dY, Y, dX, dgain, dbias, eps=1e-6):
    x, y = f64(X), f64(dY)
    g = np.ones(X.shape[-1]) if gain is None else f64(gain)
    b = np.zeros(X.shape[-1]) if bias is None else f64(bias)
    C = x.shape[-1]
    t = C / 32 + 12
    mean = x.mean(-1, keepdims=True)
    rstd = 1 / np.sqrt(((x - mean) ** 2).mean(-1, keepdims=True) + eps)
    xhat = (x - mean) * rstd
    A = np.abs(x).max(-1, keepdims=True) * rstd
    e_hat = (2 * t + 8) * U * (A + np.abs(xhat))
    ref = orc.layer_norm(x, g, b, eps)
    within("Y", Y, ref, e_hat * np.abs(g) + 4 * U * (np.abs(ref) + np.abs(b)) + HALF_STEP[dtype] * np.abs(ref))
    rx, rg, rb = orc.layer_norm_backward(x, g, y, eps)
    a = y * g
    S = rstd * (np.abs(a).max(-1, keepdims=True) + np.abs(xhat).max(-1, keepdims=True) * np.abs(a * xhat).max(-1, keepdims=True))
    within("dX", dX, rx, (4 * t + 24) * U * S * (1 + A) + HALF_STEP[dtype] * np.abs(rx))
    rows = tuple(range(x.ndim - 1))
    if dgain is not None:
        within("dgain", dgain, rg, (np.abs(y * xhat) * 64 * U + np.abs(y) * (2 * t + 8) * U * (A + np.abs(xhat))).sum(rows) + U)
        within("dbias", dbias, rb, (np.abs(y).sum(rows)) * 64 * U + U)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", [
    ((1,), 64), ((1, 12, 1), 64), ((2, 5, 37), 64), ((1000,), 64), ((33,), 1), ((7, 3), 3), ((65,), 31), ((9,), 33), ((129,), 100), ((40,), 128),
    ((77,), 256), ((50,), 257), ((31,), 511), ((20,), 512), ((300,), 768), ((19,), 777), ((64,), 1000), ((257,), 1024), ((11,), 1025), ((21,), 1280),
    ((5,), 2048), ((6,), 3001), ((4,), 4096), ((3,), 5000), ((7,), 8191), ((9,), 8192), ((30000,), 64), ((4000,), 96)])
def test_against_the_definition(dtype, rows, cols):
    X, dY = rows_of(dtype, *rows, cols, seed=cols), rows_of(dtype, *rows, cols, seed=cols + 1, offset=0.1)
    g = torch.Generator(device="cuda").manual_seed(5)
    gain, bias = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda"), 0.2 * torch.randn(cols, generator=g, device="cuda")
    Y = psk.layer_norm_fwd(X, gain, bias)
    dX, dgain, dbias = psk.layer_norm_bwd(X, gain, dY)
    check(dtype, X, gain, bias, dY, Y, dX, dgain, dbias)
    again = psk.layer_norm_bwd(X, gain, dY)
    for p, q in zip((dX, dgain, dbias), again):
        assert torch.equal(p, q)                                   # a fixed order of all sums
    plain = psk.layer_norm_fwd(X)
    only, none, none2 = psk.layer_norm_bwd(X, None, dY, params=False)
    assert none is None and none2 is None
    check(dtype, X, None, None, dY, plain, only, None, None)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_rows_and_in_place(dtype):
    B, n, H = 3, 45, 5
    proj = rows_of(dtype, B, n, 3, H, 64, seed=1)
    X = proj[:, :, 1].permute(0, 2, 1, 3)                          # [B,H,n,64] inside a projection
    dY = rows_of(dtype, B, H, n, 64, seed=2)
    gain = 1 + 0.1 * rows_of("f32", 64, seed=3)
    Y = psk.layer_norm_fwd(X, gain)
    assert Y.stride() == X.stride()
    dense = psk.layer_norm_fwd(X.contiguous(), gain)
    assert torch.equal(Y, dense)
    into = torch.empty(B, n, H, 64, dtype=X.dtype, device="cuda").transpose(1, 2)
    assert psk.layer_norm_fwd(X, gain, out=into) is into or torch.equal(into, dense)
    dX, dgain, dbias = psk.layer_norm_bwd(X, gain, dY)
    dXc, dgc, dbc = psk.layer_norm_bwd(X.contiguous(), gain, dY)
    assert torch.equal(dX, dXc)
    check(dtype, X, gain, None, dY, Y, dX, dgain, dbias)
    # what lies between the rows is left as it was
    before = proj.clone()
    psk.layer_norm_fwd(X, gain, out=X)
    assert torch.equal(X, Y) and torch.equal(proj[:, :, 0], before[:, :, 0]) and torch.equal(proj[:, :, 2], before[:, :, 2])
    Xc = before[:, :, 1].permute(0, 2, 1, 3).contiguous()
    d2 = dY.clone()
    assert torch.equal(psk.layer_norm_bwd(Xc, gain, d2, out=d2)[0], dXc) and torch.equal(d2, dXc)
    x2 = Xc.clone()
    psk.layer_norm_bwd(x2, gain, dY, out=x2)
    assert torch.equal(x2, dXc)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_off_16_bytes(dtype):
    base = rows_of(dtype, 40, 70, seed=4)
    X, dY = base[:, 3:67], rows_of(dtype, 40, 64, seed=6)          # stride 70, start 3
    gain = 1 + 0.1 * rows_of("f32", 64, seed=3)
    Y = psk.layer_norm_fwd(X, gain)
    dX, dgain, dbias = psk.layer_norm_bwd(X, gain, dY)
    check(dtype, X, gain, None, dY, Y, dX, dgain, dbias)
    expanded = dY[:1].expand(40, 64)                               # one row of dY for all
    got = psk.layer_norm_bwd(X.contiguous(), gain, expanded)
    check(dtype, X, gain, None, expanded, Y, *got)
    flat = torch.zeros(200, dtype=X.dtype, device="cuda")[1:193].view(3, 64)
    flat.copy_(X[:3])
    assert torch.equal(psk.layer_norm_fwd(flat, gain, out=torch.empty(3, 64, dtype=X.dtype, device="cuda")), psk.layer_norm_fwd(flat, gain))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,stride,start", [(1, 2, 2, 0), (300, 6, 6, 2), (77, 64, 70, 2), (50, 130, 130, 0), (40, 254, 256, 2), (31, 258, 262, 4), (20, 514, 514, 6),
                                                    (33, 1002, 1002, 0), (9, 1026, 1030, 2), (7, 2046, 2050, 0), (6, 2050, 2050, 0), (5, 4094, 4094, 2), (4, 4098, 4098, 0),
                                                    (3, 8190, 8190, 2), (2, 8192, 8194, 2), (2000, 90, 90, 0)])
def test_rows_on_two_values(dtype, rows, cols, stride, start):
    """Even columns, strides and starts that are not whole 16 bytes."""
    def make(seed, offset=0.0):
        flat = torch.zeros(start + rows * stride + 8, dtype=DT[dtype], device="cuda")
        x = flat[start:start + rows * stride].view(rows, stride)[:, :cols]
        x.copy_(rows_of(dtype, rows, cols, seed=seed, offset=offset))
        return flat, x
    (fx, X), (fd, dY), (fo, out) = make(cols), make(cols + 1, 0.1), make(3)
    gain, bias = 1 + 0.1 * rows_of("f32", cols, seed=3), rows_of("f32", cols, seed=4)
    between = torch.ones_like(fo, dtype=torch.bool)
    between[start:start + rows * stride].view(rows, stride)[:, :cols] = False
    before = fo.clone()
    Y = psk.layer_norm_fwd(X, gain, bias, out=out).clone()
    assert torch.equal(fo[between], before[between])
    dX, dgain, dbias = psk.layer_norm_bwd(X, gain, dY, out=out)
    assert torch.equal(fo[between], before[between])
    check(dtype, X, gain, bias, dY, Y, dX, dgain, dbias)


def test_large_offsets_and_constant_rows():
    # a mean a thousand times the spread; rows without any spread: eps alone is under the root
    X = rows_of("f32", 64, 768, seed=8) + 1000.0
    X[5] = 3.25
    dY = rows_of("f32", 64, 768, seed=9)
    Y = psk.layer_norm_fwd(X, None, None, 1e-5)
    dX, dgain, dbias = psk.layer_norm_bwd(X, None, dY, 1e-5)
    check("f32", X, None, None, dY, Y, dX, dgain, dbias, 1e-5)
    assert (Y[5] == 0).all()


def test_one_bad_row_stays_alone():
    X, dY = rows_of("bf16", 300, 64, seed=10), rows_of("bf16", 300, 64, seed=11)
    Y, dX = psk.layer_norm_fwd(X), psk.layer_norm_bwd(X, None, dY)[0]
    X2 = X.clone()
    X2[17] = float("nan")
    X2[200, 3] = float("inf")
    Y2, dX2 = psk.layer_norm_fwd(X2), psk.layer_norm_bwd(X2, None, dY)[0]
    keep = torch.ones(300, dtype=torch.bool, device="cuda")
    keep[[17, 200]] = False
    assert torch.equal(Y[keep], Y2[keep]) and torch.equal(dX[keep], dX2[keep])
    assert Y2[17].isnan().all() and dX2[17].isnan().all()


def test_rows_far_apart():
    # offsets that pass 32 bits: two rows 2.2e9 values apart
    big = torch.empty(2_200_000_200, dtype=torch.bfloat16, device="cuda")
    X = big.as_strided((2, 64), (2_200_000_000, 1), 40)
    X.copy_(rows_of("bf16", 2, 64, seed=12))
    dY = rows_of("bf16", 2, 64, seed=13)
    dX, dgain, dbias = psk.layer_norm_bwd(X, None, dY, out=torch.empty(2, 64, dtype=torch.bfloat16, device="cuda"))
    torch.cuda.synchronize()
    Y = psk.layer_norm_fwd(X, out=X)
    check("bf16", rows_of("bf16", 2, 64, seed=12), None, None, dY, Y, dX, dgain, dbias)


def test_captured_and_replayed():
    X, dY = rows_of("bf16", 64, 768, seed=14), rows_of("bf16", 64, 768, seed=15)
    gain = 1 + 0.1 * rows_of("f32", 768, seed=16)
    psk.layer_norm_bwd(X, gain, dY)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Y = psk.layer_norm_fwd(X, gain)
        grads = psk.layer_norm_bwd(X, gain, dY)
    X.copy_(rows_of("bf16", 64, 768, seed=17))
    g.replay()
    torch.cuda.synchronize()
    for p, q in zip((Y,) + grads, (psk.layer_norm_fwd(X, gain),) + psk.layer_norm_bwd(X, gain, dY)):
        assert torch.equal(p, q)


def test_another_stream_and_ctypes(monkeypatch):
    X, dY = rows_of("bf16", 500, 64, seed=18), rows_of("bf16", 500, 64, seed=19)
    ref = (psk.layer_norm_fwd(X),) + psk.layer_norm_bwd(X, None, dY)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = (psk.layer_norm_fwd(X),) + psk.layer_norm_bwd(X, None, dY)
    side.synchronize()
    monkeypatch.setattr(binding, "_fast", binding._NoNative())
    for p, q, r in zip(ref, got, (psk.layer_norm_fwd(X),) + psk.layer_norm_bwd(X, None, dY)):
        assert torch.equal(p, q) and torch.equal(p, r)


def test_workspace_is_the_callers():
    X, dY = rows_of("bf16", 5000, 64, seed=20), rows_of("bf16", 5000, 64, seed=21)
    need = binding.layer_norm_workspace_bytes(X)
    ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    dX, dg, db = psk.layer_norm_bwd(X, None, dY, workspace=ws[:need])
    assert (ws[need:] == 7).all()
    for p, q in zip((dX, dg, db), psk.layer_norm_bwd(X, None, dY)):
        assert torch.equal(p, q)
    with pytest.raises(psk.PskError) as e:
        psk.layer_norm_bwd(X, None, dY, workspace=ws[:need - 256])
    assert e.value.code == -5


def test_refusals():
    X = rows_of("bf16", 4, 64)
    with pytest.raises(ValueError):
        psk.layer_norm_fwd(X.half())
    with pytest.raises(ValueError):
        psk.layer_norm_fwd(X, torch.ones(63, device="cuda"))
    with pytest.raises(ValueError):
        psk.layer_norm_fwd(X, torch.ones(64, device="cuda").bfloat16())
    with pytest.raises(ValueError):
        psk.layer_norm_fwd(X.t())
    with pytest.raises(ValueError):
        psk.layer_norm_bwd(X, None, X.float())
    with pytest.raises(RuntimeError):
        psk.layer_norm_fwd(X, torch.ones(64))
    for bad, code in ((dict(X=X, eps=-1.0), -1), (dict(X=X, eps=float("nan")), -1), (dict(X=rows_of("bf16", 2, 8193)), -2), (dict(X=X[:0]), -3),
                      (dict(X=X, out=X[:1].expand(4, 64)), -3)):
        with pytest.raises(psk.PskError) as e:
            psk.layer_norm_fwd(**bad)
        assert e.value.code == code


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [64, 65, 66, 768, 4096])
@pytest.mark.parametrize("spread,eps", [(1e15, 1e-6), (1e17, 1e-6), (1e-14, 0.0), (1e-17, 0.0)])
def test_spreads_far_from_one(dtype, cols, spread, eps):
    """rstd cubed is beyond fp32 for these rows; every factor of the formulas, and their products in a fitting order, are not."""
    X, dY = rows_of(dtype, 50, cols, seed=cols + 2), rows_of(dtype, 50, cols, seed=cols + 3)
    X = (X.float() * spread).to(X.dtype)
    # gradients with a part along the rows, so that the projection's term is as large as the others
    dY = (dY.float() + X.float() / X.float().std(-1, unbiased=False, keepdim=True)).to(X.dtype)
    gain, bias = 1 + 0.1 * rows_of("f32", cols, seed=3), rows_of("f32", cols, seed=4)
    Y = psk.layer_norm_fwd(X, gain, bias, eps)
    dX, dgain, dbias = psk.layer_norm_bwd(X, gain, dY, eps)
    check(dtype, X, gain, bias, dY, Y, dX, dgain, dbias, eps)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [64, 70, 77])
def test_an_output_of_other_strides(dtype, cols):
    """Rows are worked on in the order of X's strides; an output laid out in another order gets each row in its place."""
    B, n, H = 3, 45, 5
    X, dY = rows_of(dtype, B, H, n, cols, seed=31), rows_of(dtype, B, H, n, cols, seed=32)
    gain = 1 + 0.1 * rows_of("f32", cols, seed=33)
    dense, (dXd, dgd, dbd) = psk.layer_norm_fwd(X, gain), psk.layer_norm_bwd(X, gain, dY)
    for order in ((0, 2, 1), (1, 0, 2), (2, 1, 0), (2, 0, 1)):
        shape, back = [(B, H, n)[i] for i in order], [order.index(i) for i in range(3)]
        into, dinto = (torch.empty(*shape, cols, dtype=X.dtype, device="cuda").permute(*back, 3) for _ in range(2))
        got = psk.layer_norm_fwd(X, gain, out=into)
        assert got is into
        assert torch.equal(into, dense)
        dX, dgain, dbias = psk.layer_norm_bwd(X, gain, dY, out=dinto)
        assert dX is dinto or dX.data_ptr() == dinto.data_ptr()
        assert torch.equal(dinto, dXd) and torch.equal(dgain, dgd) and torch.equal(dbias, dbd)


@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_overlap(dtype, native, monkeypatch):
    """Rows that are read may lie over one another; the results' do not."""
    if not native:
        monkeypatch.setattr(binding, "_fast", binding._NoNative())
    base = rows_of(dtype, 3, 1, 5, 64, seed=41)
    long = rows_of(dtype, 200, seed=42)
    gain = 1 + 0.1 * rows_of("f32", 64, seed=3)
    for X in (base.expand(3, 7, 5, 64), base[:1, :, :1].expand(2, 7, 5, 64), long.unfold(0, 64, 8), long.unfold(0, 64, 1)):
        dY = rows_of(dtype, *X.shape, seed=43)
        Y, (dX, dgain, dbias) = psk.layer_norm_fwd(X, gain), psk.layer_norm_bwd(X, gain, dY)
        assert Y.is_contiguous() and dX.is_contiguous()
        check(dtype, X, gain, None, dY, Y, dX, dgain, dbias)
    X = rows_of(dtype, 4, 9, 5, 64, seed=44).permute(2, 0, 1, 3)[:, 1:, ::2]             # apart, in an order of their own
    assert psk.layer_norm_fwd(X, gain).stride() == X.stride()
