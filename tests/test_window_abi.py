"""Refusals of the layer normalisation and sliding-window calls, before any launch (no GPU needed)."""
import ctypes
from ctypes import byref, c_int64, c_void_p

import pytest
import torch

import paper_2310_01655_b200 as psk
from paper_2310_01655_b200.binding import NormShape, WindowShape

FAKE = c_void_p(256)          # never read: every call below is refused


@pytest.fixture(scope="module")
def L():
    from paper_2310_01655_b200 import build
    build.build()
    return psk.lib()


def norm():
    s = (c_int64 * 3)(64 * 12, 64, 64 * 12 * 4)
    return NormShape(4, 12, 9, 64, 1, 1e-6, s, s, s)


def window():
    return WindowShape(2, 4, 2, 100, 64, 32, 2, 1, 0, 0.125, 4 * 6400, 6400, 64, 2 * 6400, 6400, 64)


def norm_calls(L, s):
    return (L.psk_layer_norm_fwd(byref(s), FAKE, FAKE, FAKE, FAKE, None),
            L.psk_layer_norm_bwd(byref(s), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None))


def window_calls(L, s):
    return (L.psk_window_attn_fwd(byref(s), *[FAKE] * 6, FAKE, 1 << 40, None), L.psk_window_attn_bwd(byref(s), *[FAKE] * 10, FAKE, 1 << 40, None),
            L.psk_window_cache_fill(byref(s), *[FAKE] * 5, None), L.psk_window_decode_step(byref(s), *[FAKE] * 7, None))


@pytest.mark.parametrize("field,value,code", [
    ("dtype", 2, -1), ("eps", -1e-9, -1), ("eps", float("nan"), -1), ("eps", float("inf"), -1), ("n0", 0, -3), ("n1", -2, -3), ("n2", 0, -3), ("cols", 0, -3),
    ("cols", 8193, -2), ("n0", 1 << 30, -3), ("zs", (64 * 12, 32, 64 * 12 * 4), -3), ("zs", (0, 64, 64 * 12 * 4), -3), ("zs", (1 << 62, 64, 64 * 12 * 4), -3), ("zs", (64 * 12, 64, 1 << 43), -3)])
def test_layer_norm(L, field, value, code):
    s = norm()
    setattr(s, field, (c_int64 * 3)(*value) if isinstance(value, tuple) else value)
    if field == "zs":
        s.ys = s.zs                       # (what the forward writes)
    assert norm_calls(L, s) == (code, code) and L.psk_layer_norm_workspace_bytes(byref(s)) == 0


def test_layer_norm_pointers(L):
    s = norm()
    need = L.psk_layer_norm_workspace_bytes(byref(s))
    assert need >= 2 * 64 * 4                 # one row of both sums at least
    assert L.psk_layer_norm_fwd(None, FAKE, FAKE, FAKE, FAKE, None) == -1
    assert L.psk_layer_norm_fwd(byref(s), None, FAKE, FAKE, FAKE, None) == -1
    assert L.psk_layer_norm_fwd(byref(s), FAKE, FAKE, FAKE, None, None) == -1
    assert L.psk_layer_norm_bwd(byref(s), FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, need, None) == -1
    assert L.psk_layer_norm_bwd(byref(s), FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, need, None) == -5
    assert L.psk_layer_norm_bwd(byref(s), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, need - 1, None) == -5
    assert L.psk_layer_norm_bwd(byref(s), FAKE, FAKE, FAKE, FAKE, None, FAKE, c_void_p(264), need, None) == -5


@pytest.mark.parametrize("field,value,code", [
    ("dtype", 7, -1), ("path", 3, -1), ("scale", 0.0, -1), ("scale", -1.0, -1), ("scale", float("nan"), -1), ("scale", float("inf"), -1),
    ("B", 0, -3), ("H", 3, -3), ("Hkv", 0, -3), ("window", 0, -3), ("window", -1, -3), ("sinks", -1, -3), ("h", 128, -2)])
def test_window(L, field, value, code):
    s = window()
    setattr(s, field, value)
    assert window_calls(L, s) == (code,) * 4
    assert L.psk_window_workspace_bytes(byref(s), 0) == 0 and L.psk_window_cache_bytes(byref(s)) == 0


@pytest.mark.parametrize("fields,code", [
    (dict(n=0), -3), (dict(n=1 << 29), -3), (dict(q_stride_n=32), -3), (dict(q_stride_h=0), -3), (dict(kv_stride_b=6400), -3), (dict(q_stride_n=68, q_stride_h=6800, q_stride_b=27200), -4),
    (dict(kv_stride_h=6401, kv_stride_b=2 * 6401), -4), (dict(q_stride_n=1 << 38), -3), (dict(path=2, dtype=0), -2)])
def test_window_rows(L, fields, code):
    s = window()
    for f, v in fields.items():
        setattr(s, f, v)
    assert window_calls(L, s)[:2] == (code, code)
    assert L.psk_window_workspace_bytes(byref(s), 1) == 0


@pytest.mark.parametrize("window,sinks,path,ok", [(32, 0, 0, True), (1 << 22, 0, 0, False), (2**31 - 1, 0, 2, False), (32, 1, 0, False), ((1 << 21) - 129, 0, 0, True),
                                                  ((1 << 21) - 128, 0, 0, False), (1 << 22, 3, 1, True)])
def test_window_longest_tiles(L, window, sinks, path, ok):
    """A tile of keys on the tensor cores is worked on for less than the second that a wait lasts at most."""
    n = 1 << 22
    s = WindowShape(1, 16, 1, n, 64, window, sinks, 1, path, 0.125, 64 * n * 16, 64 * n, 64, 64 * n, 64 * n, 64)
    assert [L.psk_window_workspace_bytes(byref(s), k) > 0 for k in (0, 1)] == [ok, ok]
    if not ok:
        assert window_calls(L, s)[:2] == (-2, -2)


def test_window_cache_too_large(L):
    s = window()
    s.window, s.sinks = 2**31 - 1, 5
    assert window_calls(L, s)[2:] == (-3, -3) and L.psk_window_cache_bytes(byref(s)) == 0


def test_window_pointers(L):
    s = window()
    fwd, bwd = (L.psk_window_workspace_bytes(byref(s), k) for k in (0, 1))
    assert fwd >= 4 and bwd >= fwd + 2 * 4 * 100 * 4 and L.psk_window_cache_bytes(byref(s)) == 2 * 2 * 34 * 64 * 2
    call = lambda k, p: L.psk_window_attn_fwd(byref(s), *[p if i == k else FAKE for i in range(6)], FAKE, fwd, None)
    for k in (0, 1, 2, 4, 5):
        assert call(k, None) == -1
    for k, off in ((0, 264), (1, 258), (2, 264), (3, 257), (4, 264), (5, 258)):
        assert call(k, c_void_p(off)) == -4
    assert L.psk_window_attn_fwd(byref(s), *[FAKE] * 6, None, fwd, None) == -5
    assert L.psk_window_attn_fwd(byref(s), *[FAKE] * 6, FAKE, fwd - 1, None) == -5
    assert L.psk_window_attn_fwd(byref(s), *[FAKE] * 6, c_void_p(272), fwd, None) == -5
    assert L.psk_window_attn_fwd(None, *[FAKE] * 6, FAKE, fwd, None) == -1
    for k in (0, 1, 2, 4, 5, 6, 7, 8, 9):
        assert L.psk_window_attn_bwd(byref(s), *[None if i == k else FAKE for i in range(10)], FAKE, bwd, None) == -1
    assert L.psk_window_attn_bwd(byref(s), *[FAKE] * 10, FAKE, fwd, None) == -5
    for k in (0, 1, 3, 4):
        assert L.psk_window_cache_fill(byref(s), *[None if i == k else FAKE for i in range(5)], None) == -1
    for k in range(7):
        assert L.psk_window_decode_step(byref(s), *[None if i == k else FAKE for i in range(7)], None) == -1
        assert L.psk_window_decode_step(byref(s), *[c_void_p(258) if i == k else FAKE for i in range(7)], None) == -4


def test_strides_of_single_extents_are_not_looked_at(L):
    s = window()
    s.B, s.H, s.Hkv, s.n = 1, 1, 1, 1
    for side in ("q", "kv"):
        for d in "bhn":
            setattr(s, "%s_stride_%s" % (side, d), 0)
    assert L.psk_window_workspace_bytes(byref(s), 0) > 0


def test_binding_refuses_cpu_tensors(L):
    x = torch.zeros(1, 2, 8, 64)
    for call in (lambda: psk.layer_norm_fwd(x), lambda: psk.layer_norm_bwd(x, None, x), lambda: psk.window_attn_fwd(x, x, x, 4),
                 lambda: psk.window_attn_bwd(x, x, x, x, x[..., 0], x, 4), lambda: psk.window_cache_fill(x, x, x, x, 8),
                 lambda: psk.window_decode_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], x, x, torch.zeros(1, dtype=torch.int32), 8)):
        with pytest.raises(RuntimeError, match="CUDA"):
            call()


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("B,H,Hkv,n,window,sinks", [(100, 24, 8, 1, 7, 2), (1, 1, 1, 1, 1, 0), (3, 12, 12, 129, 60, 0), (2, 16, 2, 5000, 300, 16), (1, 8, 1, 700, 300, 0)])
def test_the_backwards_workspace_serves_the_forward(L, dtype, B, H, Hkv, n, window, sinks):
    for path in (0, 1):
        s = WindowShape(B, H, Hkv, n, 64, window, sinks, dtype, path, 0.125, 64 * n * H, 64 * n, 64, 64 * n * Hkv, 64 * n, 64)
        fwd, bwd = (L.psk_window_workspace_bytes(byref(s), k) for k in (0, 1))
        assert 256 <= fwd <= bwd


@pytest.mark.parametrize("numbers", [dict(window=2**32 + 5), dict(window=2**31), dict(window=5, sinks=2**32), dict(window=5, sinks=2**40 + 1), dict(window=-2**32 + 5),
                                     dict(window=5, path=2**32 + 1)])
def test_numbers_beyond_32_bits(numbers):
    """A descriptor's fields would take them modulo 2^32: another window, and no error."""
    x = torch.zeros(1, 2, 8, 64)
    with pytest.raises(psk.PskError) as e:
        psk.binding.make_window_shape(x, x, **numbers)
    assert e.value.code == -3


def test_extents_beyond_32_bits():
    for x in (torch.zeros(1, 1, 1, 64).expand(2**32 + 1, 1, 1, 64), torch.zeros(1, 1, 1, 64).expand(1, 1, 2**31, 64)):
        with pytest.raises(psk.PskError) as e:
            psk.binding.make_window_shape(x, x, 5)
        assert e.value.code == -3
    s = psk.binding.make_window_shape(torch.zeros(1, 2, 8, 64), torch.zeros(1, 1, 8, 64), 2**31 - 1, 2**31 - 1)
    assert (s.window, s.sinks) == (2**31 - 1, 2**31 - 1)


@pytest.mark.parametrize("scale,code", [(3.4e38, -1), (2.4e38, -1), (2.35e38, None), (1e-45, None)])
def test_scales_at_the_ends(L, scale, code):
    """Scores are kept times log2(e): a scale whose product with that is infinite would make NaN of a score of 0."""
    s = window()
    s.scale = scale
    if code is not None:
        assert window_calls(L, s) == (code,) * 4
    assert (L.psk_window_workspace_bytes(byref(s), 0) == 0) == (code is not None)
