"""The status word of the window calls: a call clears what an earlier one left there, however many items it has."""
import pytest
import torch

import paper_2310_01655_b200 as psk
from test_gpu_window import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,B,H,n", [("bf16", 1, 1, 1), ("bf16", 1, 2, 300), ("bf16", 4, 12, 700), ("bf16", 24, 12, 300), ("bf16", 3, 12, 1100), ("f32", 2, 2, 200)])
def test_an_earlier_calls_code_does_not_stay(dtype, B, H, n):
    Q, K, V, dO = make(dtype, B, H, H, n, seed=n)
    ws = torch.zeros(psk.binding.window_workspace_bytes(psk.binding.make_window_shape(Q, K, 50, 0), True), dtype=torch.uint8, device="cuda")
    word = ws[:4].view(torch.int32)
    ref = None
    for _ in range(3):
        word.fill_(7)
        assert psk.check(ws) == -7                        # (PSK_ERR_TIMEOUT: what a wait that gave up leaves)
        O, lse = psk.window_attn_fwd(Q, K, V, 50, workspace=ws)
        assert psk.check(ws) == 0
        word.fill_(7)
        out = (O, lse) + psk.window_attn_bwd(Q, K, V, O, lse, dO, 50, workspace=ws)
        assert psk.check(ws) == 0
        ref = ref or out
        assert all(torch.equal(x, y) for x, y in zip(out, ref))
