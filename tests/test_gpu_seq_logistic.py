"""The recurrence's gates against 64 bits, each small weight to its own size."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from seq_common import dtype, f64

pytestmark = pytest.mark.gpu

# In units of 2^-24: exp2 and the reciprocal are off by at most one in the last
# place (2 units each), the product with the argument's rest, 1 + e and e s by half
# of one (1 each), the state's own products by another: 9.  Of 16-bit inputs exp
# takes an argument off by 2^-24 of itself, and log2 e by another quarter of that.
def bar(x, t):
    return (9 + (0 if t == "f32" else 1.25 * np.abs(x))) * 2.0 ** -24


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_small_weights(t):
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    x = torch.linspace(-87, 87, 20001, device="cuda").to(dtype(torch, t))
    F, x64 = x.numel(), f64(x)
    s, sn = 1 / (1 + np.exp(-x64)), 1 / (1 + np.exp(x64))
    one, zero, y, h = torch.ones_like(x), torch.zeros_like(x), torch.empty_like(x), torch.empty(1, F, device="cuda")
    v3 = lambda a: a.view(1, 1, F)  # noqa: E731
    D.dtst_recurrence(v3(x), v3(one), v3(y), h_out=h)                                     # s(-z)
    got_n = f64(h)[0]
    D.dtst_recurrence(v3(x), v3(zero), v3(y), h0=torch.ones(1, F, device="cuda"), h_out=h)  # s(z)
    got_s = f64(h)[0]
    st = torch.ones(1, 1, F, device="cuda")
    g_z, g_v, g_0 = torch.empty_like(x), torch.empty_like(x), torch.empty(1, F, device="cuda")
    D.dtst_recurrence_adj(v3(x), v3(zero), v3(zero), st, v3(g_z), v3(g_v), g_h=torch.ones(1, F, device="cuda"), g_hzero=g_0)
    for name, got, ref in (("s(-z)", got_n, sn), ("s(z)", got_s, s), ("g_hzero", f64(g_0)[0], s)):
        e = np.abs(got - ref) / ref
        say(f"  {t} {name}: up to {e.max() * 2 ** 24:.1f} units of 2^-24, {(e / bar(x64, t)).max():.2f} of the bar")
        assert (e <= bar(x64, t)).all(), name
    if t == "f32":
        for name, got, ref in (("g_v", f64(g_v), sn), ("g_z", f64(g_z), s * sn)):
            assert (np.abs(got - ref) <= (ref * 2 * bar(x64, t)) + 2.0 ** -126).all(), name
