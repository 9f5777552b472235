"""The fp64 oracle of the latent-sequence operators: gradients against central
differences, 8-bit rounding against torch's conversion, and the binding's
argument checks (no GPU needed)."""

import numpy as np
import pytest
import torch

from oracle import seq_oracle as S

D = pytest.importorskip("paper_2607_14394_amd", reason="libdtst.so not built")


def differences(f, x, g, h=1e-6):
    """sum(g * f(x)) differentiated by x, central differences (error h^2 and 1e-16 / h: about 1e-9)."""
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        p, m = x.copy(), x.copy()
        p[i] += h
        m[i] -= h
        out[i] = ((f(p) - f(m)) * g).sum() / (2 * h)
    return out


def test_norm_gradient_is_the_derivative():
    rng = np.random.RandomState(1)
    u, w, g, gs = rng.randn(3, 7), rng.randn(7), rng.randn(3, 7), rng.randn(3, 7)
    g_u, g_w = S.rms_norm_adj(g, u, w, 1e-3, gs)
    assert np.abs(g_u - gs - differences(lambda a: S.rms_norm(a, w, 1e-3)[0], u, g)).max() < 1e-7
    assert np.abs(g_w - differences(lambda a: S.rms_norm(u, a, 1e-3)[0], w, g)).max() < 1e-7


@pytest.mark.parametrize("gated", [True, False])
def test_recurrence_gradient_is_the_derivative(gated):
    rng = np.random.RandomState(2)
    B, T, F = 3, 5, 2
    z, v, o, h0 = (rng.randn(B, T, F) for _ in range(3)), None, None, rng.randn(B, F)
    z, v, o = z
    o = o if gated else None
    n = np.array([5, 0, 3])
    g, gh = rng.randn(B, T, F), rng.randn(B, F)
    y, h = S.recurrence(z, v, o, h0, n)
    assert np.array_equal(h[1, -1], h0[1]) and not y[1].any() and not y[2, 3:].any()
    g_z, g_v, g_o, g_0 = S.recurrence_adj(z, v, g, h, o, gh, n)

    def run(**k):
        a = dict(z=z, v=v, o=o, h0=h0)
        a.update(k)
        y, h = S.recurrence(a["z"], a["v"], a["o"], a["h0"], n)
        return np.concatenate([y.ravel(), h[:, -1].ravel()])

    up = np.concatenate([g.ravel(), gh.ravel()])
    for got, name in ((g_z, "z"), (g_v, "v"), (g_o, "o"), (g_0, "h0")):
        if name == "o" and not gated:
            continue
        x = dict(z=z, v=v, o=o, h0=h0)[name]
        assert np.abs(got - differences(lambda a: run(**{name: a}), x, up)).max() < 1e-7, name


def test_e4m3_rounding_is_the_types():
    rng = np.random.RandomState(3)
    v = np.concatenate([rng.randn(4000) * np.exp2(rng.uniform(-12, 7, 4000)), np.arange(-448, 449) / 2.0,
                        np.arange(-64, 65) * 2.0 ** -11, [0.0]])
    v = v[np.abs(v) <= 448].astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(S.e4m3(v), want)


def test_scales_are_the_smallest_that_fit():
    x = np.zeros((7, 300))
    x[0, :3] = [448, -1, 2]
    x[1, 128] = 449
    x[2, 299] = 2.0 ** -140
    x[3, 5] = np.inf
    x[4, 5], x[4, 6] = np.nan, 896
    x[6, 0] = 3.4e38
    q, e = S.quantise(x)
    assert e[0, 0] == 0 and e[1, 1] == 1 and e[2, 2] == -126 and e[3, 0] == 0 and e[4, 0] == 1 and not e[5].any()
    assert q.shape == (7, 384) and np.isnan(q[3, 5]) and np.isnan(q[4, 5]) and q[4, 6] == 448
    assert 224 < np.abs(q[6, 0]) <= 448


# ---- argument checks ----------------------------------------------------------

def test_shapes_of_codes_and_scales():
    assert [D.code_columns(k) for k in (1, 128, 129)] == [128, 128, 256]
    assert [D.scale_columns(k) for k in (1, 512, 513)] == [4, 4, 8]
    assert D.recurrence_states_shape(3, 129, 5) == (3, 2, 5) and D.recurrence_states_shape(3, 0, 5) == (3, 0, 5)


def status(fn, *args):
    st = fn(*args)
    return st, D.lib.dtst_last_error().decode()


P = 1 << 20  # an aligned address that no refused call reads


def norm_call(x=P, res=None, w=P * 2, s=None, y=P * 3, scale=None, rstd=None, **kw):
    f = dict(rows=4, cols=64, ld_x=64, ld_res=64, ld_sum=64, ld_y=128, ld_scale=4, x_type=1, res_type=1, y_type=1,
             eps=1e-6)
    f.update(kw)
    d = D.NORM_DESC.pack(*f.values())
    return status(D.lib.dtst_rms_norm, d, x, res, w, s, y, scale, rstd, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(rows=-1), 1, "rows"), (dict(cols=0), 1, "cols"), (dict(x_type=3), 1, "x_type"), (dict(x_type=7), 1, "x_type"),
    (dict(res_type=2), 1, "res_type"), (dict(y_type=0), 1, "y_type"), (dict(y_type=3), 1, "scale"),
    (dict(scale=P * 5), 1, "scale"), (dict(eps=-1.0), 1, "eps"), (dict(eps=float("nan")), 1, "eps"),
    (dict(eps=float("inf")), 1, "eps"), (dict(cols=32769, ld_x=32769, ld_y=40000), 2, "cols"),
    (dict(x=None), 1, "x is null"), (dict(w=None), 1, "weight"), (dict(y=None), 1, "y is null"),
    (dict(x=P + 1), 1, "aligned"), (dict(ld_x=63), 1, "stride of x"), (dict(ld_y=63), 1, "stride of y"),
    (dict(res=P * 6, ld_res=60), 1, "stride of res"), (dict(y_type=3, scale=P * 5, ld_y=120), 1, "stride of y"),
    (dict(y_type=3, scale=P * 5, ld_y=136), 1, "multiple of 16"), (dict(y_type=3, scale=P * 5 + 1), 1, "aligned"),
    (dict(y_type=3, scale=P * 5, ld_scale=5), 1, "multiple of 4"), (dict(y=P + 2), 1, "overlap"),
    (dict(y=P + 8, ld_y=64), 1, "overlap"), (dict(s=P * 3), 1, "overlap"), (dict(rows=1 << 40), 2, "rows"),
    (dict(rows=1 << 50), 1, "too large"),
])
def test_norm_refusals(kw, code, word):
    st, msg = norm_call(**kw)
    assert st == code and word in msg, (st, msg)


def test_norm_of_no_rows_is_done():
    assert norm_call(rows=0, x=None, w=None, y=None)[0] == 0


def adj_call(gy=P, u=P * 2, w=P * 3, r=P * 4, gs=None, gu=P * 5, gx=None, gw=P * 6, ws=P * 7, nws=1 << 16, **kw):
    f = dict(rows=4, cols=64, ld_g_y=64, ld_u=64, ld_g_sum=64, ld_g_u=64, ld_g_x=64, x_type=1, res_type=0, accumulate=0)
    f.update(kw)
    d = D.NORM_ADJ_DESC.pack(*f.values())
    return status(D.lib.dtst_rms_norm_adj, d, gy, u, w, r, gs, gu, gx, gw, ws, nws, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(rows=-1), 1, "rows"), (dict(cols=0), 1, "cols"), (dict(res_type=2), 1, "res_type"),
    (dict(accumulate=2), 1, "accumulate"), (dict(nws=16), 1, "workspace"), (dict(ws=None), 1, "workspace"),
    (dict(gw=None), 1, "g_weight"), (dict(r=None), 1, "rstd"), (dict(u=P + 2), 1, "aligned"),
    (dict(ld_u=63), 1, "stride of u"), (dict(gu=P * 2), 1, "overlap"), (dict(gx=P), 1, "overlap"),
    (dict(gx=P * 5), 1, "overlap"), (dict(cols=40000, ld_g_y=40000, ld_u=40000, ld_g_u=40000, nws=1 << 30), 2, "cols"),
])
def test_norm_adj_refusals(kw, code, word):
    st, msg = adj_call(**kw)
    assert st == code and word in msg, (st, msg)


def quantise_call(x=P, q=P * 2, s=P * 3, qt=None, st=None, **kw):
    f = dict(rows=4, cols=200, ld_x=200, ld_q=256, ld_scale=4, ld_qt=128, ld_scale_t=4, type=1)
    f.update(kw)
    d = D.QUANTISE_DESC.pack(*f.values())
    return status(D.lib.dtst_quantise, d, x, q, s, qt, st, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(rows=-1), 1, "rows"), (dict(cols=0), 1, "cols"), (dict(type=3), 1, "type"), (dict(s=None), 1, "together"),
    (dict(q=None), 1, "together"), (dict(q=None, s=None), 1, "null"), (dict(qt=P * 4), 1, "together"),
    (dict(ld_q=200), 1, "stride of q"), (dict(ld_q=260), 1, "multiple of 16"), (dict(q=P * 2 + 8), 1, "aligned"),
    (dict(ld_scale=6), 1, "multiple of 4"), (dict(ld_x=199), 1, "stride of x"), (dict(q=P), 1, "overlap"),
    (dict(qt=P * 2, st=P * 5), 1, "overlap"), (dict(qt=P * 6, st=P * 5, ld_qt=64), 1, "stride of qt"),
])
def test_quantise_refusals(kw, code, word):
    st, msg = quantise_call(**kw)
    assert st == code and word in msg, (st, msg)


def product_call(a=P, sa=P * 2, b=P * 3, sb=P * 4, bias=None, c=P * 5, **kw):
    f = dict(m=70, n=80, k=200, ld_a=256, ld_a_scale=4, ld_b=256, ld_b_scale=4, ld_c=80, c_type=1, accumulate=0, short_sums=0)
    f.update(kw)
    d = D.PRODUCT_DESC.pack(*f.values())
    return status(D.lib.dtst_product, d, a, sa, b, sb, bias, c, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(m=-1), 1, "m >= 0"), (dict(k=0), 1, "k >= 1"), (dict(c_type=3), 1, "c_type"), (dict(accumulate=3), 1, "accumulate"), (dict(short_sums=2), 1, "short_sums"),
    (dict(ld_a=200), 1, "stride of a"), (dict(ld_b=264), 1, "multiple of 16"), (dict(sa=None), 1, "a_scale"),
    (dict(a=P + 8), 1, "aligned"), (dict(ld_c=79), 1, "stride of c"), (dict(c=P), 1, "overlap"), (dict(c=P * 5 + 1), 1, "aligned"),
    (dict(bias=P + 1), 1, "aligned"), (dict(k=1 << 24, ld_a=1 << 24, ld_b=1 << 24, ld_a_scale=1 << 17, ld_b_scale=1 << 17, m=1, n=1,
     b=1 << 30, c=1 << 40, sa=1 << 41, sb=1 << 42), 2, "2^23"),
])
def test_product_refusals(kw, code, word):
    st, msg = product_call(**kw)
    assert st == code and word in msg, (st, msg)


def test_product_of_nothing_is_done():
    assert product_call(m=0, a=None)[0] == 0 and product_call(n=0, b=None)[0] == 0


def recur_call(z=P, v=P * 2, o=P * 3, h0=None, n=None, y=P * 4, h=None, st=None, ws=P * 8, nws=1 << 30, fn="dtst_recurrence", **kw):
    f = dict(batch=2, steps=300, features=16)
    f.update({k + "_stride": (4800, 16) for k in ("z", "v", "o", "y", "g_z", "g_v", "g_o")})
    f.update(type=1)
    f.update(kw)
    flat = []
    for x in f.values():
        flat += list(x) if isinstance(x, tuple) else [x]
    d = D.RECURRENCE_DESC.pack(*flat)
    if fn == "dtst_recurrence":
        return status(D.lib.dtst_recurrence, d, z, v, o, h0, n, y, h, st, ws, nws, None)
    gz, gv, go = kw.get("out", (P * 5, P * 6, P * 7))
    return status(D.lib.dtst_recurrence_adj, d, z, v, o, n, st, y, h0, gz, gv, go, h, ws, nws, None)


@pytest.mark.parametrize("kw,code,word", [
    (dict(batch=-1), 1, "batch"), (dict(steps=-1), 1, "steps"), (dict(type=3), 1, "type"), (dict(z=None), 1, "z is null"),
    (dict(z=P + 1), 1, "aligned"), (dict(z_stride=(4800, 15)), 1, "strides of z"), (dict(v_stride=(-4800, 16)), 1, "strides of v"),
    (dict(y_stride=(160, 16)), 1, "rows of y"), (dict(y=P), 1, "overlap"), (dict(h0=P + 2), 1, "aligned"),
    (dict(batch=1 << 40, steps=1 << 40), 1, "overflow"), (dict(nws=64), 1, "workspace"), (dict(ws=None), 1, "workspace"), (dict(o_stride=(1 << 60, 16)), 1, "too large"),
])
def test_recurrence_refusals(kw, code, word):
    st, msg = recur_call(**kw)
    assert st == code and word in msg, (st, msg)


def test_recurrence_adj_refusals():
    f = "dtst_recurrence_adj"
    assert recur_call(fn=f)[1] == "states is null"
    assert "overlap" in recur_call(fn=f, st=P * 9, y=P * 5)[1]
    st, msg = recur_call(fn=f, st=P * 9, o=None)
    assert st == 1 and "g_o" in msg


def test_recurrence_of_nothing_is_done():
    assert recur_call(batch=0, z=None)[0] == 0 and recur_call(features=0, z=None)[0] == 0


def test_binding_refuses_tensors_off_the_device():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        D.dtst_rms_norm(x, torch.ones(64), torch.empty_like(x))
    with pytest.raises(ValueError):
        D.dtst_quantise(x, *D.empty_codes(4, 64, device="cpu"))
    q, s = D.empty_codes(4, 64, device="cpu")
    with pytest.raises(ValueError):
        D.dtst_product(q, s, q, s, torch.empty(4, 4))
    z = torch.zeros(1, 4, 8)
    with pytest.raises(ValueError):
        D.dtst_recurrence(z, z, torch.empty_like(z))
