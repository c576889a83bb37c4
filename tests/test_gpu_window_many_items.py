"""Window attention on the tensor cores where a CTA works on many items: the CTAs stay and take over items that have not been started, so
barrier phases, places for operands and answers of the scheduler go round several times.  148 CTAs (296 in the forward) have 6 to 18 items
each here.  Against the definition for some heads, against calls on single sequences (few items to a CTA) for all of them."""
import pytest
import torch

import paper_2310_01655_b200 as psk
from test_gpu_window import check_heads, make, run

pytestmark = pytest.mark.gpu
B, H, N = 24, 12, 1100
# whole ones, empty ones between them, ends inside a tile and on its border
RAGGED = [N, 0, 1, 129, 0, 0, N - 1, 128, 700, 0, 1024, 5, N, 64, 0, 333, 1025, 0, 256, 900, 2, 0, N, 513]


@pytest.mark.parametrize("Hkv,window,sinks,lengths", [
    (12, 100, 0, None), (12, N, 0, None), (12, 1, 0, None), (4, 300, 0, None), (12, 64, 4, None), (4, 40, 16, None), (12, 200, 130, None),
    (12, 100, 0, RAGGED), (4, 500, 0, RAGGED), (12, 64, 4, RAGGED), (4, 300, 16, RAGGED[::-1]), (12, 90, 200, RAGGED)])
def test_many_items_to_a_cta(Hkv, window, sinks, lengths):
    Q, K, V, dO = make("bf16", B, H, Hkv, N, seed=window + sinks)
    lens = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    out = run(Q, K, V, dO, window, sinks, lengths=lens)
    for _ in range(3):
        for x, y in zip(out, run(Q, K, V, dO, window, sinks, lengths=lens)):
            assert torch.equal(x, y)
    check_heads("bf16", Q, K, V, dO, out, window, sinks, lengths=lengths, heads=[(0, 0), (B // 2, Hkv // 2), (B - 1, Hkv - 1)])
    for b in range(B):
        one = run(*(x[b:b + 1] for x in (Q, K, V, dO)), window, sinks, lengths=None if lens is None else lens[b:b + 1].clone())
        for name, x, y in zip(("O", "lse", "dQ"), one, out):
            assert torch.equal(x[0], y[b]), (name, b)
        for name, x, y in zip(("dK", "dV"), one[3:], out[3:]):
            x, y = x[0].double(), y[b].double()
            if Hkv == H:                                  # (else the query heads may be dealt to several items, in fp32 sums of other groups)
                assert torch.equal(x[:, sinks:], y[:, sinks:]), (name, b)
            # sums of the same products in fp32, in other groups: off by N u of the terms' magnitudes, N <= 3300 terms (2^-12.3), which come to less than
            # ten times a head's largest result here; then one rounding each
            assert ((x - y).abs() <= 2.0 ** -7 * y.abs() + 2.0 ** -9 * y.abs().amax((1, 2), keepdim=True)).all(), (name, b)


def test_many_items_of_one_row():
    # every item is a tile of one row
    Q, K, V, dO = make("bf16", 100, 24, 8, 1, seed=5)
    O, lse, dQ, dK, dV = run(Q, K, V, dO, 7, 2)
    s = (Q.double() * K.double().repeat_interleave(3, 1)).sum(-1) * 0.125
    assert torch.equal(O, V.repeat_interleave(3, 1)) and ((lse - s).abs() <= 2.0 ** -14 * (1 + s.abs())).all()
    want = dO.double().view(100, 8, 3, 1, 64).sum(2)
    assert ((dV.double() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -18 * dO.double().view(100, 8, 3, 1, 64).abs().sum(2)).all()


def test_many_items_captured_and_beside_one_another():
    """Replayed from a graph with other inputs, and on two streams at once."""
    sets = [make("bf16", 8, H, 4, N, seed=60 + i) for i in range(2)]
    lens = torch.tensor([N, 0, 300, N, 1, 128, 0, 777], dtype=torch.int32, device="cuda")
    step = lambda Q, K, V, dO: (lambda O, lse: (O, lse) + psk.window_attn_bwd(Q, K, V, O, lse, dO, 150, 3, lengths=lens))(*psk.window_attn_fwd(Q, K, V, 150, 3, lengths=lens))
    refs = [step(*s) for s in sets]
    torch.cuda.synchronize()
    held = [x.clone() for x in sets[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(*held)
    for s, ref in zip((sets[1], sets[0]), (refs[1], refs[0])):
        for x, y in zip(held, s):
            x.copy_(y)
        for _ in range(3):
            graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, ref))
    streams, outs = [torch.cuda.Stream() for _ in sets], [[], []]
    for _ in range(5):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                outs[i].append(step(*sets[i]))
    torch.cuda.synchronize()
    for ref, some in zip(refs, outs):
        assert all(torch.equal(x, y) for one in some for x, y in zip(one, ref))
