"""The norm's last bits: 1 / rms rounded once, the output's two products once
each, so that few 8-bit and 16-bit results go to the wrong side of an edge."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S

pytestmark = pytest.mark.gpu


# In units of 2^-24 of a value between 1 and 2 of them: rounding to nearest is off
# by 1/4 of a last place (0.5 units) on average at the binade's start and half that
# relative to the value at its end, 0.35 over uniform logarithms.  The sum of
# squares adds to 1 / rms what 16 lanes' sums in 32 bits leave: below 0.1.  The
# output adds the roundings of two products: 0.35 sqrt(3) = 0.6.  (A 32-bit sum and
# root: 0.6 and 0.76.)
@pytest.mark.parametrize("rows,cols", [(4096, 200), (4096, 512), (4096, 1000), (4096, 1536), (2048, 4096), (1024, 8000),
                                       (512, 16384), (256, 32768)])
def test_rounded_once(rows, cols):
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    g = torch.Generator(device="cuda")
    g.manual_seed(cols)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp2(3 * torch.randn((rows, 1), generator=g, device="cuda"))
    w = 1 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    y, rstd = torch.empty_like(x), torch.empty(rows, device="cuda")
    D.dtst_rms_norm(x, w, y, rstd=rstd, eps=1e-6)
    x64 = x.double()
    r64 = 1 / torch.sqrt((x64 * x64).mean(dim=1) + 1e-6)
    y64 = x64 * r64[:, None] * w.double()
    units = lambda got, ref: float(((got.double() - ref) / ref)[ref != 0].abs().mean()) * 2 ** 24  # noqa: E731
    er, ey = units(rstd, r64), units(y, y64)
    say(f"[norm] {rows} x {cols}: 1 / rms off by {er:.2f}, y by {ey:.2f} units of 2^-24 on average")
    assert er <= 0.45 and ey <= 0.7


def test_weights_and_rows_at_their_ends():
    """Infinite weights make infinities of all but zeros; rows of zeros, of small
    numbers, and of numbers whose squares' sum passes 32 bits."""
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    inf = float("inf")
    x = torch.randn(6, 700, device="cuda")
    x[1, :10] = 0
    x[2] = 0
    x[3] = 1e19 * x[3]
    x[4] = 1e-19 * x[4]
    w = torch.ones(700, device="cuda")
    w[5], w[9], w[20], w[21] = inf, -inf, 3e38, float("nan")
    y, rstd = torch.empty_like(x), torch.empty(6, device="cuda")
    D.dtst_rms_norm(x, w, y, rstd=rstd, eps=0.0)
    assert float(rstd[3]) == 0 and not y[3, :5].any()
    rows = [0, 1, 4, 5]
    with np.errstate(all="ignore"):
        ref, r = S.rms_norm(x.cpu().double().numpy(), w.cpu().double().numpy(), 0.0)
        ref = ref.astype(np.float32)[rows]
    got = y.cpu().numpy()[rows]
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(got[np.isinf(ref)], ref[np.isinf(ref)])
    ok = np.isfinite(ref)
    assert (np.abs(got[ok] - ref[ok]) <= 2.0 ** -22 * np.abs(ref[ok])).all()
    assert torch.isnan(y[2]).all() and torch.isinf(rstd[2])
    assert np.allclose(rstd.cpu().numpy()[rows], r[rows], rtol=2.0 ** -22)
    D.dtst_rms_norm(x, w, y, rstd=rstd, eps=1e-6)
    assert not y[2, :5].any() and abs(float(rstd[2]) / 1e3 - 1) <= 2.0 ** -22
