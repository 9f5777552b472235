"""The short causal convolution and its backward against the fp64 oracle: taps,
steps around the runs, odd numbers of features, types, lengths, the state in
place, strides, offsets past 32 bits, graphs, central differences."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from scan_common import empty
from seq_common import f64, near, rounded

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def inputs(torch, B, T, F, K, t, seed, lengths=None, bias=True, state=True):
    rng = np.random.RandomState(seed)
    x, xv = rounded(torch, rng.randn(B, T, 2 * F), t)
    g, gv = rounded(torch, rng.randn(B, T, F), t)
    if lengths is not None:
        for i, n in enumerate(lengths):
            x[i, max(0, n):] = float("nan")
            g[i, max(0, n):] = float("nan")
    w, wv = rounded(torch, rng.randn(K, F), "f32")
    b, bv = rounded(torch, rng.randn(F), "f32")
    s, sv = rounded(torch, rng.randn(B, K - 1, F), t)
    l, lv = rounded(torch, rng.randn(B, K - 1, F), t)
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    dev = dict(x=x[..., F:], w=w, g=g, bias=b if bias else None, state=s if state else None, last=l, lengths=n)
    val = dict(x=xv[..., F:], w=wv, g=gv, bias=bv if bias else None, state=sv if state else None, last=lv,
               lengths=None if lengths is None else np.clip(lengths, 0, T))
    return dev, val


def forward(torch, D, dev, t, silu=True, **kw):
    (B, T, F), K = dev["x"].shape, dev["w"].shape[0]
    y, last = empty(torch, t, B, T, F), empty(torch, t, B, K - 1, F)
    D.dtst_conv(dev["x"], dev["w"], y, bias=dev["bias"], state=dev["state"], state_out=last, lengths=dev["lengths"], silu=silu,
                **kw)
    return y, last


def backward(torch, D, dev, t, silu=True, ends=True, accumulate=None, **kw):
    (B, T, F), K = dev["x"].shape, dev["w"].shape[0]
    g = dict(x=empty(torch, t, B, T, F), w=empty(torch, "f32", K, F), bias=empty(torch, "f32", F),
             state=empty(torch, t, B, K - 1, F))
    if accumulate is not None:
        g["w"], g["bias"] = accumulate[0].clone(), accumulate[1].clone()
    D.dtst_conv_adj(dev["x"], dev["w"], dev["g"], g["x"], g["w"], bias=dev["bias"], g_bias=g["bias"], state=dev["state"],
                    g_state_out=dev["last"] if ends else None, g_state=g["state"], lengths=dev["lengths"], silu=silu,
                    accumulate=accumulate is not None, **kw)
    return g


def oracle(val, silu=True, ends=True):
    args = dict(bias=val["bias"], state=val["state"], lengths=val["lengths"], silu=silu)
    y, last = S.conv(val["x"], val["w"], **args)
    g = S.conv_adj(val["x"], val["w"], val["g"], g_last=val["last"] if ends else None, **args)
    return y, last, dict(zip(("x", "w", "bias", "state"), g))


def compare(torch, D, dev, val, t, silu=True, ends=True):
    y, last, g = oracle(val, silu, ends)
    gy, gl = forward(torch, D, dev, t, silu)
    near(f64(gy), y, t, "y")
    assert np.array_equal(f64(gl), last)
    got = backward(torch, D, dev, t, silu, ends)
    for k, v in got.items():
        near(f64(v), g[k], t if k in ("x", "state") else "f32", "g_" + k)
    return gy, gl, got


@pytest.mark.parametrize("K", range(1, 9))
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_taps(K, t):
    torch, D = lib()
    say(f"[conv] {K} taps {t}")
    for T in (1, 2, 7, 8, 9, 50):
        compare(torch, D, *inputs(torch, 3, T, 37, K, t, K + T), t)


@pytest.mark.parametrize("F", [1, 2, 3, 4, 5, 8, 15, 64, 100, 255, 256, 257, 520, 1100])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_features(F, t):
    torch, D = lib()
    say(f"[conv] {F} features {t}")
    compare(torch, D, *inputs(torch, 2, 21, F, 4, t, F), t)


@pytest.mark.parametrize("silu", [True, False])
@pytest.mark.parametrize("bias", [True, False])
@pytest.mark.parametrize("state", [True, False])
def test_operands_left_out(silu, bias, state):
    torch, D = lib()
    dev, val = inputs(torch, 2, 30, 40, 4, "f32", 2, bias=bias, state=state)
    compare(torch, D, dev, val, "f32", silu, ends=state)
    (B, T, F), y = dev["x"].shape, forward(torch, D, dev, "f32", silu)[0]
    again = torch.empty_like(y)
    D.dtst_conv(dev["x"], dev["w"], again, bias=dev["bias"], state=dev["state"], silu=silu)   # the state at the end not wanted
    assert torch.equal(again, y)
    g, gx, gw = backward(torch, D, dev, "f32", silu), torch.empty_like(y), torch.empty_like(dev["w"])
    D.dtst_conv_adj(dev["x"], dev["w"], dev["g"], gx, gw, bias=dev["bias"], state=dev["state"], g_state_out=dev["last"],
                    silu=silu)
    assert torch.equal(gx, g["x"]) and torch.equal(gw, g["w"])


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_lengths(t):
    torch, D = lib()
    lengths = [90, 0, 1, 2, 3, 4, 8, 17, -5, 1000, 89]
    for K in (4, 8):
        dev, val = inputs(torch, len(lengths), 90, 50, K, t, 3, lengths)
        y, _, g = compare(torch, D, dev, val, t)
        for i, n in enumerate(val["lengths"]):
            assert not y[i, n:].any() and not g["x"][i, n:].any()


def test_chunks_and_single_steps_go_on():
    torch, D = lib()
    for K in (2, 4, 8):
        dev, val = inputs(torch, 2, 60, 96, K, "bf16", 5)
        y, last, _ = compare(torch, D, dev, val, "bf16")
        for cuts in ([0, 3, 4, 40, 60], list(range(61))):
            state, out = dev["state"].clone(), torch.empty_like(y)
            for s, e in zip(cuts, cuts[1:]):
                o = torch.empty(2, e - s, 96, dtype=torch.bfloat16, device="cuda")
                D.dtst_conv(dev["x"][:, s:e], dev["w"], o, bias=dev["bias"], state=state, state_out=state)
                out[:, s:e] = o
            assert torch.equal(out, y) and torch.equal(state, last)


def test_long_sequences_in_place():
    """Several runs a sequence, the state updated in place; sums in a fixed order."""
    torch, D = lib()
    B, T, F = 2, 5000, 1030
    dev, val = inputs(torch, B, T, F, 4, "bf16", 6)
    y, last, g = oracle(val)
    for _ in range(2):
        state, got = dev["state"].clone(), empty(torch, "bf16", B, T, F)
        D.dtst_conv(dev["x"], dev["w"], got, bias=dev["bias"], state=state, state_out=state)
        near(f64(got), y, "bf16", "y")
        assert np.array_equal(f64(state), last)
    a, b = backward(torch, D, dev, "bf16"), backward(torch, D, dev, "bf16")
    for k in a:
        near(f64(a[k]), g[k], "bf16" if k in ("x", "state") else "f32", "g_" + k)
        assert torch.equal(a[k], b[k])
    twice = backward(torch, D, dev, "bf16", accumulate=(a["w"], a["bias"]))
    near(f64(twice["w"]), 2 * g["w"], "f32", "g_w twice")
    near(f64(twice["bias"]), 2 * g["bias"], "f32", "g_bias twice")


def test_steps_first_and_column_ranges():
    torch, D = lib()
    dev, val = inputs(torch, 3, 50, 41, 4, "bf16", 8)
    y, last, g = compare(torch, D, dev, val, "bf16")
    flip = lambda v: v.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    for off in (0, 7):
        out = torch.full((50, 3, 120), 5.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        D.dtst_conv(flip(dev["x"]), dev["w"], out[..., off:off + 41], bias=dev["bias"], state=dev["state"])
        D.dtst_conv_adj(flip(dev["x"]), dev["w"], flip(dev["g"]), out[..., 60 + off:101 + off], torch.empty_like(dev["w"]),
                        bias=dev["bias"], state=dev["state"], g_state_out=dev["last"])
        assert torch.equal(out[..., off:off + 41], y) and torch.equal(out[..., 60 + off:101 + off], g["x"])
        assert (out[..., :off] == 5).all() and (out[..., off + 41:60 + off] == 5).all() and (out[..., 101 + off:] == 5).all()


def test_offsets_past_32_bits():
    torch, D = lib()
    dev, val = inputs(torch, 2, 70, 40, 4, "bf16", 10)
    y, _, g = oracle(val)
    big = torch.empty((2, 70, 1 << 25), dtype=torch.bfloat16, device="cuda")   # 2^32.1 values
    x, up, out, gx = (big[..., i:i + 40] for i in (1, 50, 100, 150))
    x.copy_(dev["x"])
    up.copy_(dev["g"])
    D.dtst_conv(x, dev["w"], out, bias=dev["bias"], state=dev["state"])
    near(f64(out), y, "bf16", "y")
    gw = torch.empty_like(dev["w"])
    D.dtst_conv_adj(x, dev["w"], up, gx, gw, bias=dev["bias"], state=dev["state"], g_state_out=dev["last"])
    near(f64(gx), g["x"], "bf16", "g_x")
    near(f64(gw), g["w"], "f32", "g_w")


def test_states_past_32_bits():
    """Single steps of 2^32 values of state and more, in place, and their backward."""
    torch, D = lib()
    B, F, K, bf = 1 << 20, 640, 8, torch.bfloat16
    gen = torch.Generator(device="cuda")
    gen.manual_seed(23)
    rand = lambda *s, dt=bf: torch.randn(*s, generator=gen, device="cuda", dtype=dt)  # noqa: E731
    x, g, state, last = rand(B, 1, F), rand(B, 1, F), rand(B, K - 1, F), rand(B, K - 1, F)
    w, bias = rand(K, F, dt=torch.float32), rand(F, dt=torch.float32)
    some, cols = [0, B // 2 + 1, B - 1], [0, 77, 639]
    val = dict(x=f64(x[some]), w=f64(w), bias=f64(bias), state=f64(state[some]), g=f64(g[some]), last=f64(last[some]),
               lengths=None)
    ry, rl, rg = oracle(val)
    # the sums over all entries, of some features
    z = np.concatenate([f64(state[..., cols]), f64(x[..., cols])], axis=1)
    v = (z * f64(w)[:, cols]).sum(axis=1) + f64(bias)[cols]
    p = f64(g[:, 0, cols]) * S.logistic(v) * (1 + v * S.logistic(-v))
    g_x, g_w, g_b, g_s = (torch.empty_like(v) for v in (x, w, bias, last))
    D.dtst_conv_adj(x, w, g, g_x, g_w, bias=bias, g_bias=g_b, state=state, g_state_out=last, g_state=g_s)
    near(f64(g_x[some]), rg["x"], "bf16", "g_x")
    near(f64(g_s[some]), rg["state"], "bf16", "g_state")
    near(f64(g_w[:, cols]), (p[:, None] * z).sum(axis=0), "f32", "g_w", rms=np.sqrt(((p[:, None] * z) ** 2).sum(axis=0).mean()))
    near(f64(g_b[cols]), p.sum(axis=0), "f32", "g_bias", rms=np.sqrt((p ** 2).sum(axis=0).mean()))
    y = torch.empty_like(x)
    D.dtst_conv(x, w, y, bias=bias, state=state, state_out=state)
    near(f64(y[some]), ry, "bf16", "y")
    assert np.array_equal(f64(state[some]), rl)


def test_no_numbers_stay_where_they_are():
    """A no number reaches K steps of its feature, and nothing else."""
    torch, D = lib()
    dev, _ = inputs(torch, 1, 40, 20, 4, "f32", 11)
    dev["x"][0, 10, 3] = float("nan")
    y, _ = forward(torch, D, dev, "f32")
    bad = torch.isnan(y[0])
    assert bad[10:14, 3].all() and int(bad.sum()) == 4


def test_no_steps_and_no_sequences():
    torch, D = lib()
    dev, _ = inputs(torch, 2, 4, 10, 4, "bf16", 12)
    x0 = dev["x"][:, :0]
    last = torch.empty_like(dev["state"])
    D.dtst_conv(x0, dev["w"], x0.clone(), state=dev["state"], state_out=last)
    assert torch.equal(last, dev["state"])
    D.dtst_conv(x0, dev["w"], x0.clone(), state_out=last)
    assert not last.any()
    gw, gb = torch.full_like(dev["w"], 2.0), torch.full_like(dev["bias"], 2.0)
    D.dtst_conv_adj(x0, dev["w"], x0.clone(), x0.clone(), gw, g_bias=gb, g_state_out=dev["state"], g_state=last, accumulate=True)
    assert torch.equal(last, dev["state"]) and (gw == 2).all() and (gb == 2).all()
    e = dev["x"][:0]
    D.dtst_conv(e, dev["w"], e.clone())
    D.dtst_conv_adj(e, dev["w"], e.clone(), e.clone(), gw, g_bias=gb)
    assert not gw.any() and not gb.any()


def test_replayed():
    torch, D = lib()
    dev, val = inputs(torch, 2, 700, 130, 4, "bf16", 13)
    y, last, g = compare(torch, D, dev, val, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    for stream in (s.cuda_stream, None) * 3:
        a, b = backward(torch, D, dev, "bf16", stream=stream), forward(torch, D, dev, "bf16", stream=stream)
        torch.cuda.synchronize()
        assert all(torch.equal(a[k], g[k]) for k in g) and torch.equal(b[0], y)
    ws = torch.empty(D.dtst_conv_adj_workspace(2, 700, 130, 4), dtype=torch.uint8, device="cuda")
    out, gx, gw, state = torch.empty_like(y), torch.empty_like(y), torch.empty_like(dev["w"]), dev["state"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        D.dtst_conv_adj(dev["x"], dev["w"], dev["g"], gx, gw, bias=dev["bias"], state=dev["state"], g_state_out=dev["last"], ws=ws)
        D.dtst_conv(dev["x"], dev["w"], out, bias=dev["bias"], state=state, state_out=state)
    eager = dev["state"].clone()
    for _ in range(4):
        ws.fill_(255)
        gw.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        again = torch.empty_like(y)
        D.dtst_conv(dev["x"], dev["w"], again, bias=dev["bias"], state=eager, state_out=eager)
        assert torch.equal(out, again) and torch.equal(state, eager) and torch.equal(gx, g["x"]) and torch.equal(gw, g["w"])


def test_gradients_are_differences():
    """As the scan's: 1e-5 and third derivatives times 2e-4."""
    torch, D = lib()
    B, T, F, K, step = 1, 5, 2, 3, 2.0 ** -6
    dev, _ = inputs(torch, B, T, F, K, "f32", 15)
    dev = {k: None if v is None else v.contiguous() for k, v in dev.items()}
    got = backward(torch, D, dev, "f32")

    def f():
        y, last = forward(torch, D, dev, "f32")
        return float((y.double() * dev["g"].double()).sum() + (last.double() * dev["last"].double()).sum())

    for k in ("x", "w", "bias", "state"):
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
    dev, _ = inputs(torch, 2, 6, 10, 4, "bf16", 14)
    x, w, s, y = dev["x"], dev["w"], dev["state"], torch.empty(2, 6, 10, dtype=torch.bfloat16, device="cuda")
    D.dtst_conv(x, w, y, bias=dev["bias"], state=s, state_out=s)
    for a, k in (((x.float(), w, y), {}), ((x[0], w, y), {}), ((x, w[0], y), {}), ((x, w.half(), y), {}), ((x, w, y[:, :5]), {}),
                 ((x, w[:, :9], y), {}), ((x, w, y.float()), {}), ((x, w, y), dict(bias=dev["bias"][:9])),
                 ((x, w, y), dict(state=s[:, :2])), ((x, w, y), dict(state=s.float())), ((x, w, y), dict(state_out=s[:1])),
                 ((x, w, y), dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))), ((x.cpu(), w, y), {})):
        with pytest.raises(ValueError):
            D.dtst_conv(*a, **k)
    for a, k in (((x, w, x), {}), ((x, torch.zeros(9, 10, device="cuda"), y), {})):
        with pytest.raises(D.DtstError):
            D.dtst_conv(*a, **k)
    gw = torch.empty_like(w)
    for a, k in (((x, w, y.float(), y, gw), {}), ((x, w, y, y[:1], gw), {}), ((x, w, y, y, gw[:3]), {}),
                 ((x, w, y, y, gw), dict(g_bias=dev["bias"].half())), ((x, w, y, y, gw), dict(g_state=s[:, :1]))):
        with pytest.raises(ValueError):
            D.dtst_conv_adj(*a, **k)
    for a, k in (((x, w, y, y, gw), {}), ((x, w, y, y.clone(), w), {}),
                 ((x, w, y, y.clone(), gw), dict(state=s, g_state=s)),
                 ((x, w, y, y.clone(), gw), dict(ws=torch.empty(16, dtype=torch.uint8, device="cuda")))):
        with pytest.raises(D.DtstError):
            D.dtst_conv_adj(*a, **k)
