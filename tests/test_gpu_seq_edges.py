"""Edges of the latent-sequence operators' calls: nothing to work on, many rows."""

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


@pytest.mark.parametrize("rows,cols", [((1 << 22) + 5, 8), ((1 << 22) + 1, 1030)])
def test_norm_of_millions_of_rows(rows, cols):
    """One of 65536 sequences of 64 steps and more: 2^22 rows are one launch."""
    torch, D = lib()
    x = torch.randn(rows, cols, dtype=torch.float32, device="cuda").to(torch.bfloat16)
    w, y = torch.ones(cols, device="cuda"), torch.empty_like(x)
    say(f"[norm] {rows} x {cols}")
    D.dtst_rms_norm(x, w, y)
    few = torch.empty_like(x[:1000])
    for at in (0, 1 << 20, rows - 1000):
        D.dtst_rms_norm(x[at:at + 1000], w, few)
        assert torch.equal(y[at:at + 1000], few), at
    u = x[-1000:].double()
    assert ((y[-1000:].double() - u / torch.sqrt((u * u).mean(dim=1, keepdim=True) + 1e-6)).abs() <= 2.0 ** -8 * y[-1000:].double().abs() + 1e-5).all()
