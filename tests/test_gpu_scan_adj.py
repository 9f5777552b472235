"""The state-space scan's backward against the fp64 oracle: numbers of states,
steps, features, types, lengths, operands left out, several segments, strides,
gradients added to, offsets past 32 bits, graphs, central differences."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from scan_common import SPANS, divided, empty, inputs
from seq_common import f64, near, rounded

pytestmark = pytest.mark.gpu

OPERANDS = ("x", "delta", "a", "b", "c")


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def run(torch, D, dev, t, g_y, g_h, accumulate=None, **kw):
    """Gradients into arrays of no numbers (delta's, b's and c's side by side)."""
    B, T, F = dev["x"].shape
    N = dev["a"].shape[0]
    st = empty(torch, "f32", *D.scan_states_shape(B, T, F, N))
    y = torch.empty_like(dev["x"])
    args = [dev[k] for k in OPERANDS]
    D.dtst_scan(*args, y, d=dev["d"], o=dev["o"], h0=dev["h0"], lengths=dev["lengths"], states=st)
    p = empty(torch, t, B, T, F + 2 * N)
    g = dict(x=empty(torch, t, B, T, F), delta=p[..., :F], b=p[..., F:F + N], c=p[..., F + N:], a=empty(torch, "f32", N, F),
             h0=empty(torch, "f32", B, N, F), d=None if dev["d"] is None else empty(torch, "f32", F),
             o=None if dev["o"] is None else empty(torch, t, B, T, F))
    if accumulate:
        g["a"], g["d"] = (None if v is None else v.clone() for v in accumulate)
    D.dtst_scan_adj(*args, g_y, st, *(g[k] for k in ("x", "delta", "a", "b", "c")), d=dev["d"], g_d=g["d"], o=dev["o"],
                    g_o=g["o"], g_h=g_h, g_hzero=g["h0"], lengths=dev["lengths"], accumulate=accumulate is not None, **kw)
    return g


def gradient(torch, dev, t, seed, lengths=None):
    B, T, F = dev["x"].shape
    rng = np.random.RandomState(seed + 1000)
    g, gv = rounded(torch, rng.randn(B, T, F), t)
    if lengths is not None:
        for i, n in enumerate(lengths):
            g[i, max(0, n):] = float("nan")
    h, hv = rounded(torch, rng.randn(B, *dev["a"].shape), "f32")
    return g, gv, h, hv


def compare(torch, D, dev, val, t, seed, g_h=True, **kw):
    g, gv, h, hv = gradient(torch, dev, t, seed, val["lengths"])
    ry, rh = S.scan(**val)
    gv = np.where(np.isnan(gv), 0, gv)
    want = S.scan_adj(*(val[k] for k in OPERANDS), gv, rh, val["d"], val["o"], hv if g_h else None, val["lengths"])
    got = run(torch, D, dev, t, g, h if g_h else None, **kw)
    for k, v in got.items():
        if v is not None:
            near(f64(v), want[k], "f32" if k in ("a", "d", "h0") else t, "g_" + k)
    return got, want


@pytest.mark.parametrize("N", [1, 2, 5, 16, 17, 33, 64])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_numbers_of_states(N, t):
    torch, D = lib()
    say(f"[scan_adj] {N} states {t}")
    compare(torch, D, *inputs(torch, 2, 100, 70, N, t, N), t, N)


@pytest.mark.parametrize("N,F", [(16, 260), (20, 300), (24, 260), (25, 260), (32, 260), (33, 300), (40, 200), (48, 130), (64, 300)])
def test_states_of_several_waves(N, F):
    """Workgroups of four, two and one waves: what their states take of the LDS."""
    torch, D = lib()
    say(f"[scan_adj] {N} states, {F} features")
    compare(torch, D, *inputs(torch, 2, 70, F, N, "bf16", N), "bf16", N)


@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(seed):
    torch, D = lib()
    rng = np.random.RandomState(seed)
    B, T, F, N = rng.randint(1, 5), rng.randint(1, 260), rng.randint(1, 330), rng.randint(1, 40)
    t = ("f32", "bf16", "f16")[seed % 3]
    lengths = rng.randint(0, T + 1, B) if seed % 2 else None
    say(f"[scan_adj] {B} x {T} x {F}, {N} states, {t}, lengths {lengths}")
    dev, val = inputs(torch, B, T, F, N, t, seed, lengths, gated=seed % 4 < 2, skip=seed % 3 > 0, h0=seed % 5 > 0)
    for v in val.values():
        if v is not None and np.issubdtype(np.asarray(v).dtype, np.floating):
            np.nan_to_num(v, copy=False)
    compare(torch, D, dev, val, t, seed)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 64, 65, 128, 129, 300, 700])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_steps(T, t):
    torch, D = lib()
    say(f"[scan_adj] {T} steps {t}")
    compare(torch, D, *inputs(torch, 2, T, 33, 4, t, T), t, T)


@pytest.mark.parametrize("F", [1, 3, 63, 64, 65, 130, 300])
def test_features(F):
    torch, D = lib()
    say(f"[scan_adj] {F} features")
    compare(torch, D, *inputs(torch, 3, 70, F, 6, "f32", F), "f32", F)


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("skip", [True, False])
@pytest.mark.parametrize("h0", [True, False])
def test_operands_left_out(gated, skip, h0):
    torch, D = lib()
    for T in (5, 200):
        compare(torch, D, *inputs(torch, 2, T, 40, 8, "f32", T, gated=gated, skip=skip, h0=h0), "f32", T, g_h=h0)


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_lengths(t):
    torch, D = lib()
    lengths = [300, 0, 1, 63, 64, 65, 299, 128, -5, 1000, 37]
    dev, val = inputs(torch, len(lengths), 300, 50, 7, t, 3, lengths)
    val["lengths"] = np.clip(lengths, 0, 300)
    for v in val.values():
        if v is not None and np.issubdtype(np.asarray(v).dtype, np.floating):
            np.nan_to_num(v, copy=False)
    got, _ = compare(torch, D, dev, val, t, 3)
    for i, n in enumerate(val["lengths"]):
        for k in ("x", "delta", "b", "c", "o"):
            assert not got[k][i, n:].any(), (i, k)


def test_all_lengths_zero():
    torch, D = lib()
    dev, val = inputs(torch, 3, 200, 50, 4, "f32", 4, [0, 0, 0])
    g, _, h, _ = gradient(torch, dev, "f32", 4)
    got = run(torch, D, dev, "f32", g, h)
    assert torch.equal(got["h0"], h)
    for k in ("x", "delta", "a", "b", "c", "d", "o"):
        assert not got[k].any(), k


def test_one_segment():
    """Enough entries that no sequence is divided: g_hzero comes from the spans."""
    torch, D = lib()
    dev, val = inputs(torch, 1024, 66, 130, 2, "f32", 5)
    assert D.dtst_scan_workspace(1024, 66, 130, 2) == 0
    g, gv, h, hv = gradient(torch, dev, "f32", 5)
    got = run(torch, D, dev, "f32", g, h)
    some = [0, 511, 1023]
    part = {k: v if k in ("a", "d") or v is None else v[some] for k, v in val.items()}
    want = S.scan_adj(*(part[k] for k in OPERANDS), gv[some], S.scan(**part)[1], part["d"], part["o"], hv[some])
    for k in ("x", "delta", "b", "c", "o", "h0"):
        near(f64(got[k])[some], want[k], "f32", "g_" + k)
    again = run(torch, D, dev, "f32", g, h)
    assert all(torch.equal(got[k], again[k]) for k in got)   # a fixed order of sums


def test_many_segments():
    torch, D = lib()
    dev, val = inputs(torch, 1, 3000, 100, 3, "f32", 6)
    got, _ = compare(torch, D, dev, val, "f32", 6)
    g, _, h, _ = gradient(torch, dev, "f32", 6)
    again = run(torch, D, dev, "f32", g, h)
    assert all(torch.equal(got[k], again[k]) for k in got)


@pytest.mark.parametrize("case", SPANS, ids=lambda c: "x".join(map(str, c[:4])) + "-" + c[4])
def test_segments_of_several_spans(case):
    """Some entries have a gradient, so that the sums over all are those of some; the
    others' are zero."""
    torch, D = lib()
    B, T, F, N, t, lengths, _, segments = case
    got = divided(D, B, T, F, N)
    assert got[1] == segments and 2 * segments <= got[2] + 1
    say(f"[scan_adj] {B} x {T} x {F}, {N} states, {t}: {segments} segments of {got[2]} spans")
    dev, val = inputs(torch, B, T, F, N, t, 31, lengths)
    g, gv, h, hv = gradient(torch, dev, t, 31, lengths)
    some = sorted({0, B // 3, B // 2, B - 1})
    rest = [i for i in range(B) if i not in some]
    g[rest], h[rest] = 0, 0
    part = {k: v if k in ("a", "d") or v is None else np.asarray(v)[some] for k, v in val.items()}
    for v in part.values():
        if v is not None and np.issubdtype(v.dtype, np.floating):
            np.nan_to_num(v, copy=False)
    want = S.scan_adj(*(part[k] for k in OPERANDS), np.nan_to_num(gv[some]), S.scan(**part)[1], part["d"], part["o"],
                      hv[some], part["lengths"])
    out = run(torch, D, dev, t, g, h)
    for k, v in out.items():
        if k in ("a", "d"):
            near(f64(v), want[k], "f32", "g_" + k)
        else:
            near(f64(v)[some], want[k], "f32" if k == "h0" else t, "g_" + k)
            assert not v[rest].any(), k
    if lengths is not None:
        for i, n in enumerate(lengths):
            for k in ("x", "delta", "b", "c", "o"):
                assert not out[k][i, n:].any(), (i, k)
    ws = torch.full((D.dtst_scan_adj_workspace(B, T, F, N),), 255, dtype=torch.uint8, device="cuda")
    again = run(torch, D, dev, t, g, h, ws=ws)
    assert all(torch.equal(out[k], again[k]) for k in out)   # a fixed order of sums


def test_added_to_and_in_place():
    torch, D = lib()
    dev, val = inputs(torch, 2, 150, 70, 5, "bf16", 7)
    g, gv, h, hv = gradient(torch, dev, "bf16", 7)
    want = S.scan_adj(*(val[k] for k in OPERANDS), gv, S.scan(**val)[1], val["d"], val["o"], hv)
    once = run(torch, D, dev, "bf16", g, h)
    twice = run(torch, D, dev, "bf16", g, h, accumulate=(once["a"], once["d"]))
    for k in ("a", "d"):
        near(f64(twice[k]), 2 * want[k], "f32", "g_" + k)
    st = torch.empty(D.scan_states_shape(2, 150, 70, 5), device="cuda")
    D.dtst_scan(*(dev[k] for k in OPERANDS), torch.empty_like(dev["x"]), h0=dev["h0"], states=st)
    state = h.clone()   # g_hzero in g_h's place, d's gradient not wanted
    out = [torch.empty_like(dev[k]) for k in OPERANDS]
    D.dtst_scan_adj(*(dev[k] for k in OPERANDS), g, st, out[0], out[1], out[2], out[3], out[4], d=dev["d"], o=dev["o"],
                    g_o=torch.empty_like(dev["x"]), g_h=state, g_hzero=state)
    near(f64(state), want["h0"], "f32", "g_h0")
    assert torch.equal(out[2], once["a"])


def test_offsets_past_32_bits():
    torch, D = lib()
    dev, val = inputs(torch, 2, 70, 40, 4, "bf16", 10)
    g, gv, h, hv = gradient(torch, dev, "bf16", 10)
    want = S.scan_adj(*(val[k] for k in OPERANDS), gv, S.scan(**val)[1], val["d"], val["o"], hv)
    big = torch.empty((2, 70, 1 << 25), dtype=torch.bfloat16, device="cuda")   # 2^32.1 values
    at = 0

    def place(v):
        nonlocal at
        r = big[..., at:at + v.shape[2]]
        r.copy_(v)
        at += v.shape[2]
        return r

    for k in ("x", "delta", "o", "b", "c"):
        dev[k] = place(dev[k])
    st = torch.empty(D.scan_states_shape(2, 70, 40, 4), device="cuda")
    D.dtst_scan(*(dev[k] for k in OPERANDS), place(dev["x"]), d=dev["d"], o=dev["o"], h0=dev["h0"], states=st)
    g = place(g)
    o = {k: place(dev[k]) for k in ("x", "delta", "b", "c", "o")}
    o["a"], o["d"] = torch.empty_like(dev["a"]), torch.empty_like(dev["d"])
    D.dtst_scan_adj(*(dev[k] for k in OPERANDS), g, st, *(o[k] for k in OPERANDS), d=dev["d"], g_d=o["d"], o=dev["o"],
                    g_o=o["o"], g_h=h)
    for k, v in o.items():
        near(f64(v), want[k], "f32" if k in "ad" else "bf16", "g_" + k)


def test_column_ranges_leave_the_rest():
    torch, D = lib()
    dev, val = inputs(torch, 2, 70, 37, 3, "bf16", 8)
    g, _, h, _ = gradient(torch, dev, "bf16", 8)
    want = run(torch, D, dev, "bf16", g, h)
    st = torch.empty(D.scan_states_shape(2, 70, 37, 3), device="cuda")
    D.dtst_scan(*(dev[k] for k in OPERANDS), torch.empty_like(dev["x"]), d=dev["d"], o=dev["o"], h0=dev["h0"], states=st)
    w = torch.full((70, 2, 131), 5.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)   # steps first
    out = dict(x=w[..., 1:38], delta=w[..., 40:77], b=w[..., 79:82], c=w[..., 82:85], o=w[..., 90:127])
    ga, gd = torch.empty_like(dev["a"]), torch.empty_like(dev["d"])
    D.dtst_scan_adj(*(dev[k] for k in OPERANDS), g, st, out["x"], out["delta"], ga, out["b"], out["c"], d=dev["d"], g_d=gd,
                    o=dev["o"], g_o=out["o"], g_h=h)
    for k, v in out.items():
        assert torch.equal(v, want[k]), k
    assert torch.equal(ga, want["a"]) and torch.equal(gd, want["d"])
    for s in (slice(0, 1), slice(38, 40), slice(77, 79), slice(85, 90), slice(127, 131)):
        assert (w[..., s] == 5).all()


def test_no_steps_and_no_sequences():
    torch, D = lib()
    dev, _ = inputs(torch, 2, 4, 10, 3, "f32", 12)
    h = torch.randn(2, 3, 10, device="cuda")
    for cut in (lambda v: v[:, :0], lambda v: v[:0]):
        e = {k: cut(dev[k]) for k in ("x", "delta", "b", "c", "o")}
        B = e["x"].shape[0]
        ga, gd, g0 = torch.full_like(dev["a"], 2.0), torch.full_like(dev["d"], 2.0), torch.empty(B, 3, 10, device="cuda")
        st = torch.empty(D.scan_states_shape(B, e["x"].shape[1], 10, 3), device="cuda")
        call = lambda **kw: D.dtst_scan_adj(e["x"], e["delta"], dev["a"], e["b"], e["c"], e["x"].clone(), st,  # noqa: E731
                                            e["x"].clone(), e["x"].clone(), ga, e["b"].clone(), e["c"].clone(), d=dev["d"],
                                            g_d=gd, o=e["o"], g_o=e["x"].clone(), g_h=h[:B], g_hzero=g0, **kw)
        call(accumulate=True)
        assert (ga == 2).all() and (gd == 2).all() and torch.equal(g0, h[:B])
        call()
        assert not ga.any() and not gd.any()


@pytest.mark.parametrize("B,T,F,N", [(2, 700, 130, 5), (1, 90, 300, 64)])
def test_replayed(B, T, F, N):
    """A backward captured and replayed, with eager work between, and two streams in turns."""
    torch, D = lib()
    dev, val = inputs(torch, B, T, F, N, "bf16", 13)
    g, _, h, _ = gradient(torch, dev, "bf16", 13)
    want = run(torch, D, dev, "bf16", g, h)
    st = torch.empty(D.scan_states_shape(B, T, F, N), device="cuda")
    args = [dev[k] for k in OPERANDS]
    D.dtst_scan(*args, torch.empty_like(dev["x"]), d=dev["d"], o=dev["o"], h0=dev["h0"], states=st)

    def call(ws=None, stream=None):
        r = dict(x=torch.empty_like(dev["x"]), delta=torch.empty_like(dev["x"]), a=torch.empty_like(dev["a"]),
                 b=torch.empty(B, T, N, dtype=torch.bfloat16, device="cuda"),
                 c=torch.empty(B, T, N, dtype=torch.bfloat16, device="cuda"), d=torch.empty_like(dev["d"]),
                 o=torch.empty_like(dev["x"]), h0=torch.empty_like(h))
        D.dtst_scan_adj(*args, g, st, *(r[k] for k in OPERANDS), d=dev["d"], g_d=r["d"], o=dev["o"], g_o=r["o"], g_h=h,
                        g_hzero=r["h0"], ws=ws, stream=stream)
        return r

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    rs = [call(stream=k) for k in (s.cuda_stream, None) * 3]
    torch.cuda.synchronize()
    for r in rs:
        assert all(torch.equal(r[k], want[k]) for k in r)
    ws = torch.empty(D.dtst_scan_adj_workspace(B, T, F, N), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        r = call(ws)
    for _ in range(4):
        ws.fill_(255)
        for v in r.values():
            v.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(r[k], want[k]) for k in r)
        call()


def test_gradients_are_differences():
    """Central differences of the 32-bit forward: its 2^-22 or so over twice the step
    of 2^-6 leaves 1e-5 of a value of some units, the step's own square 2e-4 times
    third derivatives of some units."""
    torch, D = lib()
    B, T, F, N, step = 1, 5, 3, 2, 2.0 ** -6
    dev, _ = inputs(torch, B, T, F, N, "f32", 15)
    dev = {k: None if v is None else v.contiguous() for k, v in dev.items()}
    g, _, h, _ = gradient(torch, dev, "f32", 15)
    got = run(torch, D, dev, "f32", g, h)

    def f():
        y, last = torch.empty(B, T, F, device="cuda"), torch.empty(B, N, F, device="cuda")
        D.dtst_scan(*(dev[k] for k in OPERANDS), y, d=dev["d"], o=dev["o"], h0=dev["h0"], h_out=last)
        return float((y.double() * g.double()).sum() + (last.double() * h.double()).sum())

    for k in ("x", "delta", "a", "b", "c", "d", "o", "h0"):
        for i in np.ndindex(*dev[k].shape):
            at = float(dev[k][i])
            dev[k][i] = at + step
            up = f()
            dev[k][i] = at - step
            down = f()
            dev[k][i] = at
            assert abs((up - down) / (2 * step) - float(got[k][i])) < 1e-2, (k, i)


def test_refusals():
    torch, D = lib()
    dev, _ = inputs(torch, 2, 6, 10, 3, "bf16", 14)
    bf = torch.bfloat16
    z, n3 = torch.zeros(2, 6, 10, dtype=bf, device="cuda"), torch.zeros(2, 6, 3, dtype=bf, device="cuda")
    st = torch.zeros(D.scan_states_shape(2, 6, 10, 3), device="cuda")
    good = dict({k: dev[k] for k in OPERANDS}, g_y=z, states=st, g_x=z.clone(), g_delta=z.clone(), g_a=dev["a"].clone(),
                g_b=n3, g_c=n3.clone(), d=dev["d"], g_d=dev["d"].clone(), o=dev["o"], g_o=z.clone())

    def call(**kw):
        D.dtst_scan_adj(**dict(good, **kw))

    call()
    for bad in (dict(x=dev["x"].float()), dict(g_y=z.float()), dict(states=st[..., :9]), dict(states=st.double()),
                dict(g_x=z[:, :5]), dict(g_a=dev["a"].half()), dict(g_a=dev["a"].t().contiguous().t()), dict(g_b=n3.float()),
                dict(g_c=n3[..., :2]), dict(g_d=dev["d"][:9]), dict(o=None), dict(g_o=None), dict(g_h=st), dict(g_hzero=dev["a"]),
                dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")), dict(ws=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call(**bad)
    for bad in (dict(g_x=z), dict(g_b=n3, g_c=n3), dict(g_a=dev["a"]), dict(d=None), dict(g_delta=dev["delta"]),
                dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(D.DtstError):
            call(**bad)
