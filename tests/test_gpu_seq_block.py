"""The operators of a block one after the other, each against 64 bits on the
values that it was given.

End to end a block has jumps: the norm's output rounds to 8 bits and the gates to
bf16.  A value that lies at a rounding's edge goes to either side by the last
bit of a 32-bit sum, and a gate a bf16 step apart moves the state by 1e-3 of
itself: two correct 32-bit paths differ by that in a last state, now and then.
So every operator's result is checked where it is made, the roundings as
roundings, and the states on the gates that the product gave."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from seq_common import f64

pytestmark = pytest.mark.gpu


def rounds_to(got, ref, step, slack):
    """Whether got, multiples of `step`, are ref rounded to nearest, to either
    side where ref is within `slack` of an edge."""
    return (np.abs(got - ref) <= step / 2 + slack).all()


@pytest.mark.parametrize("B,T,W,F,lengths", [(2, 300, 1536, 2048, None), (3, 140, 640, 322, [140, 0, 77]), (4, 1, 2048, 2048, None),
                                             (1, 2048, 1000, 130, None)])
def test_operator_by_operator(B, T, W, F, lengths):
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    R, bf = B * T, torch.bfloat16
    g = torch.Generator(device="cuda")
    say(f"[block] {B} x {T} x {W}, {F} features, lengths {lengths}")

    def run(seed):
        g.manual_seed(seed)
        r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        x, res = (r(R, W) * torch.exp2(r(R, 1))).to(bf), r(R, W) * torch.exp2(r(R, 1))
        w, h0 = 1 + 0.2 * r(W), r(B, F)
        w1, w2 = D.empty_codes(3 * F, W), D.empty_codes(W, F)
        D.dtst_quantise(r(3 * F, W) / W ** 0.5, *w1)
        D.dtst_quantise(r(W, F) / F ** 0.5, *w2)
        bias = torch.cat([2 + 0.1 * r(F), 0.1 * r(2 * F)])
        n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        u, q, yq = torch.empty_like(res), D.empty_codes(R, W), D.empty_codes(R, F)
        p, y, c, h = (torch.full(s, float("nan"), dtype=t, device="cuda") for s, t in
                      (((B, T, 3 * F), bf), ((B, T, F), bf), ((R, W), bf), ((B, F), torch.float32)))
        D.dtst_rms_norm(x, w, q[0], res=res, sum_out=u, scale=q[1], eps=1e-6)
        D.dtst_product(*q, *w1, p.view(R, 3 * F), bias=bias)
        D.dtst_recurrence(p[..., :F], p[..., F:2 * F], y, o=p[..., 2 * F:], h0=h0, h_out=h, lengths=n)
        D.dtst_quantise(y.view(R, F), *yq)
        D.dtst_product(*yq, *w2, c)
        return dict(x=x, res=res, w=w, h0=h0, w1=w1, w2=w2, bias=bias, u=u, q=q, p=p, y=y, h=h, yq=yq, c=c)

    a, _, b = run(1), run(2), run(1)
    for k in ("u", "p", "y", "h", "c"):
        assert torch.equal(a[k], b[k]), k           # (the same again, others in between)
    values = lambda q: S.values(q[0].float().cpu().numpy(), q[1].view(torch.uint8).cpu().numpy()[:, :q[0].shape[1] // 128].astype(int) - 127)  # noqa: E731
    # the sum, exactly; the norm's codes: rounded from within 2^-21 of the value (its mean, root and
    # two products are each off by a few 2^-24)
    assert torch.equal(a["u"], a["x"].float() + a["res"])
    y64, _ = S.rms_norm(f64(a["u"]), f64(a["w"]), 1e-6)
    pad = (-W) % 128
    y64 = np.pad(y64, ((0, 0), (0, pad)))
    got = values(a["q"])
    sc = np.exp2(np.repeat(a["q"][1].view(torch.uint8).cpu().numpy()[:, :(W + pad) // 128].astype(float) - 127, 128, axis=1))
    top = np.repeat(np.abs(y64).reshape(R, -1, 128).max(axis=2), 128, axis=1)
    assert (top <= 448 * sc * (1 + 2.0 ** -21)).all() and (top >= 224 * sc * (1 - 2.0 ** -21)).all()
    v = np.minimum(np.abs(y64) / sc, 448)
    step = np.exp2(np.maximum(np.floor(np.log2(np.maximum(v, 2.0 ** -9))), -6) - 3) * sc
    assert rounds_to(got, np.sign(y64) * v * sc, step, 2.0 ** -21 * np.abs(y64))
    # the first product on these codes, with its bias
    w1 = values(a["w1"])
    p64 = S.product(got, w1, f64(a["bias"]))
    size = np.sqrt((got ** 2).sum(axis=1)[:, None] * (w1 ** 2).sum(axis=1)[None, :]) + np.abs(f64(a["bias"]))
    gp = f64(a["p"]).reshape(R, 3 * F)
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(p64), 2.0 ** -120))) - 7)
    assert rounds_to(gp, p64, step, 2.0 ** -21 * size)
    # the states on these gates
    p = f64(a["p"])
    ry, rh = S.recurrence(p[..., :F], p[..., F:2 * F], p[..., 2 * F:], f64(a["h0"]), lengths)
    off = np.linalg.norm(f64(a["h"]) - rh[:, -1]) / np.linalg.norm(rh[:, -1])
    say(f"  last states: rel {off:.1e}")
    assert off <= 1e-6
    one = max(1.0, np.abs(rh).max())
    assert (np.abs(f64(a["y"]) - ry) <= 2.0 ** -8 * np.abs(ry) + 2e-6 * one).all()
    # y's codes, exactly, and the second product on them
    yq, e = S.quantise(f64(a["y"]).reshape(R, F))
    assert np.array_equal(values(a["yq"]), S.values(yq, e))
    w2, yv = values(a["w2"]), S.values(yq, e)
    c64 = S.product(yv, w2)
    size = np.sqrt((yv ** 2).sum(axis=1)[:, None] * (w2 ** 2).sum(axis=1)[None, :])
    step = np.exp2(np.floor(np.log2(np.maximum(np.abs(c64), 2.0 ** -120))) - 7)
    assert rounds_to(f64(a["c"]), c64, step, 2.0 ** -21 * size)
