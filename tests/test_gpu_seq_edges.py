"""Edges of the latent-sequence operators' calls: nothing to work on."""

import pytest

from gpu_common import say, torch_gpu

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("cols", [1, 300, 5000, 32768])
def test_norm_backward_of_no_rows(cols, accumulate):
    """No array of rows is there, nor a weight: the weight's gradient is zero, or stays."""
    torch, D = lib()
    n = D.dtst_rms_norm_adj_workspace(0, cols)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")    # (no numbers)
    g_w = torch.randn(cols, device="cuda")
    want = g_w.clone() if accumulate else torch.zeros_like(g_w)
    d = D.NORM_ADJ_DESC.pack(0, cols, cols, cols, cols, cols, cols, 0, 0, accumulate)
    say(f"[norm backward] 0 x {cols}, accumulate {accumulate}")
    st = D.lib.dtst_rms_norm_adj(d, None, None, None, None, None, None, None, g_w.data_ptr(), ws.data_ptr(), n,
                                 D.torch_stream())
    assert st == 0, D.lib.dtst_last_error()
    assert torch.equal(g_w, want)
