"""Calls of the latent-sequence operators on two streams at once, each with the
workspace that the binding takes for it."""

import numpy as np
import pytest

from gpu_common import torch_gpu
from oracle import seq_oracle as S
from seq_common import f64, near, rounded

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def test_a_workspace_is_none_that_the_current_stream_has_freed():
    torch, D = lib()
    s, dev = torch.cuda.Stream(), torch.device("cuda", torch.cuda.current_device())
    for n in (4096, 3 << 20, 40 << 20):
        old = torch.empty(n, dtype=torch.uint8, device=dev)
        p, size = old.data_ptr(), old.nbytes
        del old
        q, m, ws = D._scratch(None, n, dev, s.cuda_stream)
        assert q + m <= p or q >= p + size
    torch.cuda.synchronize()


def test_two_streams_in_turns():
    """Every call has an output of its own that starts as no number."""
    torch, D = lib()
    B, T, F, R, C = 2, 3000, 200, 700, 513
    rng = np.random.RandomState(1)
    z, zv = rounded(torch, rng.randn(B, T, F) * 2 + 1.5, "bf16")
    v, vv = rounded(torch, rng.randn(B, T, F), "bf16")
    g, gv = rounded(torch, rng.randn(R, C), "f32")
    u, uv = rounded(torch, rng.randn(R, C), "f32")
    w, wv = rounded(torch, 1 + 0.1 * rng.randn(C), "f32")
    nan = lambda *shape, dtype=torch.float32: torch.full(shape, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    y0, rstd, g_u = torch.empty_like(u), nan(R), torch.empty_like(u)
    D.dtst_rms_norm(u, w, y0, rstd=rstd, eps=1e-6)
    ys = [nan(B, T, F, dtype=torch.bfloat16) for _ in range(12)]
    gws = [nan(C) for _ in range(12)]
    gus = [torch.empty_like(u) for _ in range(2)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for i in range(0, 12, 2):
        for k, stream in enumerate((s.cuda_stream, None)):
            D.dtst_recurrence(z, v, ys[i + k], stream=stream)
            D.dtst_rms_norm_adj(g, u, w, rstd, gus[k], gws[i + k], stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, ys[0]) for a in ys) and all(torch.equal(a, gws[0]) for a in gws)
    near(f64(ys[0]), S.recurrence(zv, vv)[0], "bf16", "y")
    near(f64(gws[0]), S.rms_norm_adj(gv, uv, wv, 1e-6)[1], "f32", "g_w")
