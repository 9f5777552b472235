"""Infinite states and gradients in the recurrence: they stay while the gates
are above zero, however small the product of many gates is, and become no number
at a gate that is zero, as one step after the other has it."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from seq_common import f64, rounded

pytestmark = pytest.mark.gpu


def alike(got, ref, name, tol=1e-5):
    """Infinities and no numbers in the same places, the others near."""
    assert np.array_equal(np.isnan(got), np.isnan(ref)), name
    inf = np.isinf(ref)
    assert np.array_equal(np.where(inf, ref, 0), np.where(np.isinf(got), got, 0)), name
    ok = np.isfinite(ref)
    d = np.abs(got[ok] - ref[ok])
    assert d.size == 0 or (d <= tol * np.maximum(1, np.abs(ref[ok]).max())).all(), name


# F: the first feature meets an infinite first state, the second an infinite input
# at some step, the third both signs, the fourth a closed gate, the rest none; the
# last feature counts put two features in a lane
@pytest.mark.parametrize("B,F", [(2, 6), (70, 130)])
@pytest.mark.parametrize("T", [1, 16, 100, 128, 129, 300, 700])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.filterwarnings("ignore::RuntimeWarning")
def test_infinite_states(B, F, T, gated):
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    rng = np.random.RandomState(T)
    # gates of e^-2 to e^-6: a wave's product is above zero, a span's is not
    z, v, o = rng.uniform(-6, -2, (B, T, F)), rng.randn(B, T, F), rng.uniform(0.5, 2, (B, T, F))
    h0, gh = rng.randn(B, F), rng.randn(B, F)
    g = rng.uniform(0.5, 2, (B, T, F))
    h0[:, 0] = np.inf
    gh[:, 0] = -np.inf
    v[:, T // 3, 1] = -np.inf
    h0[:, 2], v[:, T // 2, 2] = np.inf, -np.inf
    h0[:, 3], z[:, T // 2, 3] = np.inf, -np.inf
    gh[:, 3] = np.inf
    z[:, T // 4, 4] = -np.inf
    (z, zv), (v, vv), (o, ov), (h0, hv), (gh, ghv), (g, gv) = (rounded(torch, a, "f32") for a in (z, v, o, h0, gh, g))
    say(f"[infinite] {B} x {T} x {F}, gated {gated}")
    new = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    y, h, st = new(B, T, F), new(B, F), new(*D.recurrence_states_shape(B, T, F))
    kw = dict(o=o) if gated else {}
    D.dtst_recurrence(z, v, y, h0=h0, h_out=h, states=st, **kw)
    ry, rh = S.recurrence(zv, vv, ov if gated else None, hv)
    alike(f64(y), ry, "y")
    alike(f64(h), rh[:, -1], "h")
    alike(f64(st), rh[:, 0:T:D.RECURRENCE_SPAN], "states")
    gz, gvv, go, g0 = new(B, T, F), new(B, T, F), new(B, T, F), new(B, F)
    D.dtst_recurrence_adj(z, v, g, st, gz, gvv, g_h=gh, g_hzero=g0, **(dict(o=o, g_o=go) if gated else {}))
    rz, rv, ro, r0 = S.recurrence_adj(zv, vv, gv, rh, ov if gated else None, ghv)
    alike(f64(gvv), rv, "g_v")
    alike(f64(gz), rz, "g_z")
    alike(f64(g0), r0, "g_hzero")
    if gated:
        alike(f64(go), ro, "g_o")
