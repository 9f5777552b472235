"""RMS norm with the residual's addition, its backward, and 8-bit rows, against
the fp64 oracle: row lengths around every kernel form's limits, the types,
strides and odd offsets, updates in place, zeros and values that are no
numbers."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from seq_common import dtype, f64, near, outside, rounded, strided

pytestmark = pytest.mark.gpu

TYPES = [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")]
COLS = [1, 7, 64, 127, 128, 129, 500, 512, 513, 1024, 1025, 1537, 2048, 2049, 4096, 4097, 8192, 8200, 16384, 16385,
        32767, 32768]


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def codes_near(torch, D, q, s, v, name):
    """Codes and scales of the values v: each within half a code's step, the
    scale the smallest that fits, the padding as documented."""
    r, k = v.shape
    kb = -(-k // 128)
    qv, sb = q.float().cpu().double().numpy(), s.view(torch.uint8).cpu().numpy().astype(np.int64)
    assert not qv[:, k:].any() and (sb[:, kb:] == 127).all(), f"{name}: padding"
    _, want = S.quantise(v)
    low, high = S.quantise(v * (1 - 1e-5))[1], S.quantise(v * (1 + 1e-5))[1]
    e = sb[:, :kb] - 127
    assert ((e == want) | (e == low) | (e == high)).all(), f"{name}: scales"
    sc = np.repeat(np.exp2(e.astype(np.float64)), 128, axis=1)[:, :k]
    with np.errstate(divide="ignore"):
        step = np.exp2(np.maximum(np.floor(np.log2(np.abs(v) / sc)), -6) - 3) * sc
    off = np.abs(qv[:, :k] * sc - v) - step / 2 - 1e-5 * np.abs(v)
    say(f"  {name}: codes differ by up to {np.abs(qv[:, :k] * sc - v).max():.2e}")
    assert (off <= 0).all(), f"{name}: {int((off > 0).sum())} codes off"


def inputs(torch, rows, cols, tx, tr, seed, res=True):
    rng = np.random.RandomState(seed)
    x, xv = rounded(torch, rng.randn(rows, cols) * np.exp2(rng.uniform(-3, 3, (rows, 1))), tx)
    r, rv = rounded(torch, rng.randn(rows, cols), tr) if res else (None, 0.0)
    w, wv = rounded(torch, 1 + 0.3 * rng.randn(cols), "f32")
    # the sum in fp32, then the residual's type: what the norm is of
    u = np.float32(xv) + np.float32(rv)
    return x, r, w, wv, rounded(torch, u, tr)[1]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("tx,tr", TYPES)
def test_norm(cols, tx, tr):
    torch, D = lib()
    rows = 5
    x, r, w, wv, u = inputs(torch, rows, cols, tx, tr, cols)
    say(f"[norm] {rows} x {cols} {tx} {tr}")
    s, y = torch.empty_like(r), torch.empty_like(x)
    rstd = torch.empty(rows, device="cuda")
    D.dtst_rms_norm(x, w, y, res=r, sum_out=s, rstd=rstd, eps=1e-5)
    yv, rv = S.rms_norm(u, wv, 1e-5)
    assert np.array_equal(f64(s), u)
    near(f64(y), yv, tx, "y")
    near(f64(rstd), rv, "f32", "rstd")
    q, sc = D.empty_codes(rows, cols)
    D.dtst_rms_norm(x, w, q, res=r, sum_out=s, scale=sc, eps=1e-5)
    assert np.array_equal(f64(s), u)
    codes_near(torch, D, q, sc, yv, "codes")


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("tx,tr", TYPES)
def test_norm_adj(cols, tx, tr):
    torch, D = lib()
    rows = 11
    rng = np.random.RandomState(cols + 1)
    _, _, w, wv, _ = inputs(torch, rows, cols, tx, tr, cols)
    u, uv = rounded(torch, rng.randn(rows, cols), tr)
    g, gv = rounded(torch, rng.randn(rows, cols), tx)
    gs, gsv = rounded(torch, rng.randn(rows, cols), tr)
    say(f"[norm_adj] {rows} x {cols} {tx} {tr}")
    rstd = torch.from_numpy(S.rms_norm(uv, wv, 1e-5)[1]).float().cuda()
    g_u, g_x, g_w = torch.empty_like(u), torch.empty_like(g), torch.full_like(w, 3.0)
    D.dtst_rms_norm_adj(g, u, w, rstd, g_u, g_w, g_sum=gs, g_x=g_x)
    ru, rw = S.rms_norm_adj(gv, uv, wv, 1e-5, gsv)
    near(f64(g_u), ru, tr, "g_u")
    near(f64(g_x), ru, tx, "g_x")
    near(f64(g_w), rw, "f32", "g_w")
    # added to, without the other gradient, in place of it
    D.dtst_rms_norm_adj(g, u, w, rstd, gs, g_w, g_sum=gs, accumulate=True)
    near(f64(gs), ru, tr, "g_u in place")
    near(f64(g_w), 2 * rw, "f32", "g_w twice")
    D.dtst_rms_norm_adj(g, u, w, rstd, g_u, g_w)
    # relative to the terms t rstd of the difference: with one column it all but
    # cancels (t rstd^3 eps), below what the rounding of rstd to 32 bits moves it by
    terms = gv * wv * S.rms_norm(uv, wv, 1e-5)[1][:, None]
    near(f64(g_u), S.rms_norm_adj(gv, uv, wv, 1e-5)[0], tr, "g_u alone", rms=np.sqrt((terms ** 2).mean()))


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 9, 64, 1000, 8193])
def test_rows(rows):
    torch, D = lib()
    cols = 384
    x, r, w, wv, u = inputs(torch, rows, cols, "bf16", "bf16", rows)
    y, s, rstd = torch.empty_like(x), torch.empty_like(r), torch.empty(rows, device="cuda")
    D.dtst_rms_norm(x, w, y, res=r, sum_out=s, rstd=rstd)
    near(f64(y), S.rms_norm(u, wv, 1e-6)[0], "bf16", "y")
    g, gv = rounded(torch, np.random.RandomState(rows).randn(rows, cols), "bf16")
    g_u, g_w, g_w2 = torch.empty_like(s), torch.empty_like(w), torch.empty_like(w)
    D.dtst_rms_norm_adj(g, s, w, rstd, g_u, g_w)
    ru, rw = S.rms_norm_adj(gv, u, wv, 1e-6)
    near(f64(g_u), ru, "bf16", "g_u")
    near(f64(g_w), rw, "f32", "g_w")
    D.dtst_rms_norm_adj(g, s, w, rstd, g_u, g_w2)
    assert torch.equal(g_w, g_w2)   # a fixed order of sums


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_column_ranges_at_any_alignment(t, offset):
    torch, D = lib()
    rows, cols = 6, 333
    x, r, w, wv, u = inputs(torch, rows, cols, t, t, 5)
    xs, _ = strided(torch, x, 6, offset)
    rs, _ = strided(torch, r, 2, offset)
    yb = strided(torch, x, 4, offset)
    sb = strided(torch, x, 1, offset)
    D.dtst_rms_norm(xs, w, yb[0], res=rs, sum_out=sb[0])
    near(f64(yb[0]), S.rms_norm(u, wv, 1e-6)[0], t, "y")
    assert np.array_equal(f64(sb[0]), u)
    assert outside(yb[1], cols, offset) and outside(sb[1], cols, offset)
    q, sc = D.empty_codes(rows, cols)
    D.dtst_quantise(xs, q, sc)
    qv, e = S.quantise(f64(x))
    assert np.array_equal(q.float().cpu().double().numpy(), qv)


def test_updates_in_place():
    torch, D = lib()
    x, r, w, wv, u = inputs(torch, 7, 640, "bf16", "f32", 8)
    D.dtst_rms_norm(x, w, x, res=r, sum_out=r)
    assert np.array_equal(f64(r), u)
    near(f64(x), S.rms_norm(u, wv, 1e-6)[0], "bf16", "y")
    x, _, w, wv, u = inputs(torch, 7, 640, "f16", "f16", 9, res=False)
    D.dtst_rms_norm(x, w, x)
    near(f64(x), S.rms_norm(u, wv, 1e-6)[0], "f16", "y without a residual")


def test_rows_of_zeros_and_of_no_numbers():
    torch, D = lib()
    x = torch.randn(4, 300, device="cuda")
    x[0] = 0
    x[1, 7] = float("nan")
    x[2, 9] = float("inf")
    w = torch.ones(300, device="cuda")
    y, q = torch.empty_like(x), D.empty_codes(4, 300)
    D.dtst_rms_norm(x, w, y, eps=1e-6)
    assert not y[0].any() and torch.isnan(y[1]).all() and torch.isfinite(y[3]).all()
    assert torch.isnan(y[2, 9]) and not y[2, :9].any()          # 1 / rms is zero
    D.dtst_rms_norm(x, w, q[0], scale=q[1], eps=1e-6)
    v = q[0].float()
    assert not v[0].any() and torch.isnan(v[1, :300]).all() and not v[1, 300:].any() and torch.isfinite(v[3]).all()
    D.dtst_rms_norm(x[:1], w, y[:1], eps=0.0)                   # 0 / 0
    assert torch.isnan(y[0]).all()
    n = torch.empty(0, 300, device="cuda")
    D.dtst_rms_norm(n, w, torch.empty_like(n))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (3, 129), (127, 64), (128, 128), (129, 300), (257, 513),
                                       (640, 1000), (5, 4096)])
def test_quantise(rows, cols, t):
    torch, D = lib()
    rng = np.random.RandomState(rows + cols)
    v = rng.randn(rows, cols) * np.exp2(rng.uniform(-12, 4, (rows, 1)))
    v[rng.rand(rows, cols) < 0.1] = 0
    if rows > 2:
        v[2] = 0
    x, xv = rounded(torch, v, t)
    say(f"[quantise] {rows} x {cols} {t}")
    for which in ("rows", "cols", "both"):
        q, s = D.empty_codes(rows, cols)
        qt, st = D.empty_codes(cols, rows)
        if which == "rows":
            D.dtst_quantise(x, q, s)
        elif which == "cols":
            D.dtst_quantise(x, qt=qt, scale_t=st)
        else:
            D.dtst_quantise(x, q, s, qt=qt, scale_t=st)
        for a, (cq, cs), on in ((xv, (q, s), "rows"), (xv.T, (qt, st), "cols")):
            if which in (on, "both"):
                want, e = S.quantise(a)
                kb = e.shape[1]
                sb = cs.view(torch.uint8).cpu().numpy().astype(np.int64)
                assert np.array_equal(cq.float().cpu().double().numpy(), want), (which, on)
                assert np.array_equal(sb[:, :kb] - 127, e) and (sb[:, kb:] == 127).all(), (which, on)


def test_quantise_extremes():
    torch, D = lib()
    x = torch.zeros(6, 256, device="cuda")
    x[0, 0], x[0, 1] = 448.0, -447.9
    x[1, 0], x[1, 1] = 448.00003, 1.0
    x[2, 0] = 2.0 ** -140
    x[3, 0], x[3, 1], x[3, 2], x[3, 200] = float("inf"), float("nan"), 5.0, 3.4e38
    x[4, 5] = -float("inf")
    want, e = S.quantise(x.cpu().double().numpy())
    q, s = D.empty_codes(6, 256)
    D.dtst_quantise(x, q, s)
    assert np.array_equal(q.float().cpu().double().numpy(), want, equal_nan=True)
    assert np.array_equal(s.view(torch.uint8).cpu().numpy()[:, :2].astype(int) - 127, e)


def test_rows_past_32_bits():
    torch, D = lib()
    rows, cols, ld = 300, 200, 1 << 24      # 300 rows 2^24 apart: over 2^32 elements
    x, r, w, wv, u = inputs(torch, rows, cols, "bf16", "bf16", 12)
    big = torch.empty((rows, ld), dtype=torch.bfloat16, device="cuda")
    xs, ys = big[:, 5:5 + cols], big[:, 1000:1000 + cols]
    xs.copy_(x)
    D.dtst_rms_norm(xs, w, ys, res=r)
    near(f64(ys), S.rms_norm(u, wv, 1e-6)[0], "bf16", "y")
    q, s = D.empty_codes(rows, cols)
    D.dtst_quantise(xs, q, s)
    assert np.array_equal(q.float().cpu().double().numpy(), S.quantise(f64(x))[0])
