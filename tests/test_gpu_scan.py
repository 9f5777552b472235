"""The state-space scan against the fp64 oracle: numbers of states around every
kernel form, steps around a span and a segment, odd numbers of features, types,
lengths, states in place, strides, offsets past 32 bits, infinities, graphs."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from scan_common import SPANS, divided, empty, inputs
from seq_common import dtype, f64, near, rounded

pytestmark = pytest.mark.gpu

# The arithmetic of a step adds a few units of 2^-24 to each term c h; the states
# add up steps that decay, and an exponent's product with a rounds once: relative
# to the terms' sizes below 1e-6 each, 1e-5 (near's bar, relative to the RMS) for
# the sums over 64 states.


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def run(torch, D, dev, t, kept=False, **kw):
    B, T, F = dev["x"].shape
    N = dev["a"].shape[0]
    y, h = empty(torch, t, B, T, F), empty(torch, "f32", B, N, F)
    st = empty(torch, "f32", *D.scan_states_shape(B, T, F, N)) if kept else None
    D.dtst_scan(dev["x"], dev["delta"], dev["a"], dev["b"], dev["c"], y, d=dev["d"], o=dev["o"], h0=dev["h0"], h_out=h,
                lengths=dev["lengths"], states=st, **kw)
    return y, h, st


def compare(torch, D, dev, val, t, kept=True):
    y, h, st = run(torch, D, dev, t, kept)
    ry, rh = S.scan(**val)
    near(f64(y), ry, t, "y")
    near(f64(h), rh[:, -1], "f32", "h")
    if kept:
        near(f64(st), rh[:, :-1:D.SCAN_SPAN], "f32", "states")
    return y, h, st


@pytest.mark.parametrize("N", [1, 2, 5, 8, 9, 16, 17, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_numbers_of_states(N, t):
    torch, D = lib()
    say(f"[scan] {N} states {t}")
    compare(torch, D, *inputs(torch, 2, 150, 70, N, t, N), t)


@pytest.mark.parametrize("F", [70, 230])
@pytest.mark.parametrize("N", [3, 4, 7, 12, 13, 16, 20, 24, 32, 36, 40, 41, 48, 52, 56, 57, 64])
def test_every_form(N, F):
    """Each number of states that a kernel is built for, and one with states left out,
    by workgroups of one wave and of four, which share b and c; two segments."""
    torch, D = lib()
    say(f"[scan] {N} states, {F} features")
    for t, lengths in (("f32", None), ("bf16", [77, 0, 5]), ("f16", [1, 20, 80])):
        compare(torch, D, *inputs(torch, 3, 80, F, N, t, N, lengths), t)


@pytest.mark.parametrize("seed", range(12))
def test_random_shapes(seed):
    torch, D = lib()
    rng = np.random.RandomState(100 + seed)
    B, T, F, N = rng.randint(1, 5), rng.randint(1, 400), rng.randint(1, 330), rng.randint(1, 65)
    t = ("f32", "bf16", "f16")[seed % 3]
    lengths = rng.randint(0, T + 1, B) if seed % 2 else None
    say(f"[scan] {B} x {T} x {F}, {N} states, {t}, lengths {lengths}")
    dev, val = inputs(torch, B, T, F, N, t, seed, lengths, gated=seed % 4 < 2, skip=seed % 3 > 0, h0=seed % 5 > 0)
    compare(torch, D, dev, val, t)


@pytest.mark.parametrize("T", [1, 2, 7, 8, 9, 31, 32, 33, 63, 64, 65, 128, 129, 500, 1100])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_steps(T, t):
    torch, D = lib()
    say(f"[scan] {T} steps {t}")
    compare(torch, D, *inputs(torch, 2, T, 33, 4, t, T), t)


@pytest.mark.parametrize("F", [1, 3, 63, 64, 65, 255, 256, 257, 600])
@pytest.mark.parametrize("t", ["f32", "f16"])
def test_features(F, t):
    torch, D = lib()
    say(f"[scan] {F} features {t}")
    compare(torch, D, *inputs(torch, 3, 70, F, 6, t, F), t)


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("skip", [True, False])
@pytest.mark.parametrize("h0", [True, False])
def test_operands_left_out(gated, skip, h0):
    torch, D = lib()
    for T in (5, 200):
        compare(torch, D, *inputs(torch, 2, T, 40, 8, "f32", T, gated=gated, skip=skip, h0=h0), "f32")


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_lengths(t):
    torch, D = lib()
    lengths = [300, 0, 1, 63, 64, 65, 299, 128, -5, 1000, 37]
    dev, val = inputs(torch, len(lengths), 300, 50, 7, t, 3, lengths)
    val["lengths"] = np.clip(lengths, 0, 300)
    y, h, st = compare(torch, D, dev, val, t)
    assert not y[1].any() and torch.equal(h[1], dev["h0"][1]) and torch.equal(st[1, -1], dev["h0"][1])
    dev, val = inputs(torch, 3, 300, 50, 7, t, 4, [0, 0, 0])
    y, h, _ = run(torch, D, dev, t)
    assert not y.any() and torch.equal(h, dev["h0"])


def test_chunks_and_single_steps_go_on():
    """A sequence at once, in chunks, and step by step, the state updated in place."""
    torch, D = lib()
    dev, val = inputs(torch, 2, 200, 96, 16, "f32", 5)
    y, h, _ = compare(torch, D, dev, val, "f32")
    for cuts in ([0, 64, 65, 130, 200], list(range(201))):
        state, out = dev["h0"].clone(), torch.empty_like(y)
        for s, e in zip(cuts, cuts[1:]):
            part = {k: v if k in ("a", "d") else v[:, s:e] for k, v in dev.items() if k not in ("h0", "lengths")}
            o = torch.empty(2, e - s, 96, device="cuda")
            D.dtst_scan(part["x"], part["delta"], part["a"], part["b"], part["c"], o, d=part["d"], o=part["o"], h0=state,
                        h_out=state)
            out[:, s:e] = o
        near(f64(out), S.scan(**val)[0], "f32", "y")
        near(f64(state), f64(h), "f32", "h")


def test_many_segments_in_place():
    """The state that enters is that which leaves, while other segments still run."""
    torch, D = lib()
    dev, val = inputs(torch, 1, 5000, 130, 3, "f32", 6)
    assert D.dtst_scan_workspace(1, 5000, 130, 3) > 0
    ry, rh = S.scan(**val)
    for _ in range(3):
        state, y = dev["h0"].clone(), empty(torch, "f32", 1, 5000, 130)
        D.dtst_scan(dev["x"], dev["delta"], dev["a"], dev["b"], dev["c"], y, d=dev["d"], o=dev["o"], h0=state, h_out=state)
        near(f64(y), ry, "f32", "y")
        near(f64(state), rh[:, -1], "f32", "h")


@pytest.mark.parametrize("case", SPANS, ids=lambda c: "x".join(map(str, c[:4])) + "-" + c[4])
def test_segments_of_several_spans(case):
    torch, D = lib()
    B, T, F, N, t, lengths, segments, _ = case
    got = divided(D, B, T, F, N)
    assert got[0] == segments and 2 * segments <= got[2] + 1
    say(f"[scan] {B} x {T} x {F}, {N} states, {t}: {segments} segments of {got[2]} spans")
    dev, val = inputs(torch, B, T, F, N, t, 21, lengths)
    y, h, st = run(torch, D, dev, t, True)
    some = sorted({0, B // 3, B // 2, B - 1})
    part = {k: v if k in ("a", "d") or v is None else np.asarray(v)[some] for k, v in val.items()}
    ry, rh = S.scan(**part)
    near(f64(y)[some], ry, t, "y")
    near(f64(h)[some], rh[:, -1], "f32", "h")
    near(f64(st)[some], rh[:, :-1:D.SCAN_SPAN], "f32", "states")
    if lengths is not None:
        for i, n in enumerate(lengths):
            assert not y[i, n:].any(), i
    # the states updated in place, with the workspace full of no numbers
    state, y2 = dev["h0"].clone(), torch.empty_like(y)
    ws = torch.full((D.dtst_scan_workspace(B, T, F, N),), 255, dtype=torch.uint8, device="cuda")
    D.dtst_scan(dev["x"], dev["delta"], dev["a"], dev["b"], dev["c"], y2, d=dev["d"], o=dev["o"], h0=state, h_out=state,
                lengths=dev["lengths"], ws=ws)
    assert torch.equal(y2, y) and torch.equal(state, h)


def test_infinite_states_through_segments_of_several_spans():
    """As test_infinite_states_and_no_numbers, where a segment's decay comes from the sum
    of several spans' steps: below the smallest number, though no step's is."""
    torch, D = lib()
    B, T, F, N = 8, 300, 4096, 16
    assert divided(D, B, T, F, N)[0] == 5
    dev, _ = inputs(torch, B, T, F, N, "f32", 22, gated=False)
    dev["a"][:, :] = -16.0
    dev["h0"][2, 0, 3] = float("inf")
    dev["x"][2, 100, 5] = float("nan")
    dev["c"][:] = dev["c"].abs() + 0.1
    y, h, _ = run(torch, D, dev, "f32")
    assert torch.isinf(h[2, 0, 3]) and torch.isfinite(h[2, 1, 3]) and torch.isinf(y[2, :, 3]).all()
    assert torch.isnan(h[2, :, 5]).all() and torch.isnan(y[2, 100:, 5]).all() and torch.isfinite(y[2, :100, 5]).all()
    ok = torch.ones(F, dtype=torch.bool, device="cuda")
    ok[3] = ok[5] = False
    assert torch.isfinite(y[2][:, ok]).all() and torch.isfinite(y[:2]).all() and torch.isfinite(y[3:]).all()


def test_states_past_2_gib():
    """Single steps of 2^29 values of state, in place, and their backward."""
    torch, D = lib()
    B, F, N = 2048, 4096, 64
    gen = torch.Generator(device="cuda")
    gen.manual_seed(23)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, delta, g = rand(B, 1, F), rand(B, 1, F), rand(B, 1, F)
    b, c, a, d = rand(B, 1, N), rand(B, 1, N), -torch.exp(rand(N, F)), rand(F)
    h, g_h = rand(B, N, F), rand(B, N, F)
    y, st = empty(torch, "f32", B, 1, F), empty(torch, "f32", B, 1, N, F)
    some, cols = [0, 1023, 2047], [0, 77, 4095]
    val = {k: f64(v[some]) for k, v in dict(x=x, delta=delta, b=b, c=c, h0=h).items()}
    val.update(a=f64(a), d=f64(d))
    ry, rh = S.scan(**val)
    hv, gv = f64(h[:, :, cols]), f64(g_h[:, :, cols])
    D.dtst_scan(x, delta, a, b, c, y, d=d, h0=h, h_out=h, states=st)
    near(f64(y[some]), ry, "f32", "y")
    near(f64(h[some]), rh[:, -1], "f32", "h")
    near(f64(st[some, 0]), rh[:, 0], "f32", "states")
    out = [torch.empty_like(v) for v in (x, delta, a, b, c, d)]
    want = S.scan_adj(val["x"], val["delta"], val["a"], val["b"], val["c"], f64(g[some]), rh, val["d"], None, f64(g_h[some]))
    D.dtst_scan_adj(x, delta, a, b, c, g, st, *out[:5], d=d, g_d=out[5], g_h=g_h, g_hzero=g_h)
    for k, v in (("x", out[0]), ("delta", out[1]), ("b", out[3]), ("c", out[4]), ("h0", g_h)):
        near(f64(v[some]), want[k], "f32", "g_" + k)
    # the sums over all entries, of some features: relative to the terms' size times the root of their number
    xv, dv, yv = (f64(v[:, 0, cols]) for v in (x, delta, g))
    step = np.logaddexp(0.0, dv)[:, None]
    terms = step * np.exp(step * f64(a)[:, cols]) * (yv[:, None] * f64(c)[:, 0, :, None] + gv) * hv
    near(f64(out[2][:, cols]), terms.sum(axis=0), "f32", "g_a", rms=np.sqrt((terms ** 2).sum(axis=0).mean()))
    near(f64(out[5][cols]), (yv * xv).sum(axis=0), "f32", "g_d", rms=np.sqrt(B))


def test_entries_past_one_segment():
    """More waves than the card holds: sequences are not divided."""
    torch, D = lib()
    B, T, F, N = 128, 66, 1024, 2
    assert D.dtst_scan_workspace(B, T, F, N) == 0
    dev, val = inputs(torch, B, T, F, N, "bf16", 7)
    y, h, _ = run(torch, D, dev, "bf16")
    some = [0, 63, 127]
    ry, rh = S.scan(**{k: v if k in ("a", "d") or v is None else v[some] for k, v in val.items()})
    near(f64(y)[some], ry, "bf16", "y")
    near(f64(h)[some], rh[:, -1], "f32", "h")


def test_steps_first_and_column_ranges():
    """(steps, batch) order and outputs between other columns, which stay."""
    torch, D = lib()
    dev, val = inputs(torch, 3, 90, 40, 4, "bf16", 8)
    want, h, _ = compare(torch, D, dev, val, "bf16")
    flip = lambda v: v.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    for wide, off in ((120, 0), (121, 7)):
        out = torch.full((90, 3, wide), 5.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
        y = out[..., off:off + 40]
        D.dtst_scan(flip(dev["x"]), flip(dev["delta"]), dev["a"], flip(dev["b"]), flip(dev["c"]), y, d=dev["d"],
                    o=flip(dev["o"]), h0=dev["h0"])
        assert torch.equal(y, want)
        assert (out[..., :off] == 5).all() and (out[..., off + 40:] == 5).all()


def test_groups_of_features_are_calls_on_their_columns():
    torch, D = lib()
    dev, val = inputs(torch, 2, 80, 96, 4, "f32", 9)
    y, h = empty(torch, "f32", 2, 80, 96), empty(torch, "f32", 2, 4, 96)
    for g in range(3):
        c = slice(32 * g, 32 * g + 32)
        hg = torch.empty(2, 4, 32, device="cuda")
        D.dtst_scan(dev["x"][..., c], dev["delta"][..., c], dev["a"][:, c].contiguous(), dev["b"], dev["c"], y[..., c],
                    d=dev["d"][c], o=dev["o"][..., c], h0=dev["h0"][..., c].contiguous(), h_out=hg)
        h[..., c] = hg
    ry, rh = S.scan(**val)
    near(f64(y), ry, "f32", "y")
    near(f64(h), rh[:, -1], "f32", "h")


def test_offsets_past_32_bits():
    torch, D = lib()
    dev, val = inputs(torch, 2, 70, 40, 4, "bf16", 10)
    big = torch.empty((2, 70, 1 << 25), dtype=torch.bfloat16, device="cuda")   # 2^32.1 values
    at = 0
    for k in ("x", "delta", "o", "b", "c"):
        v = big[..., at:at + dev[k].shape[2]]
        v.copy_(dev[k])
        dev[k], at = v, at + dev[k].shape[2]
    y = big[..., at:at + 40]
    D.dtst_scan(dev["x"], dev["delta"], dev["a"], dev["b"], dev["c"], y, d=dev["d"], o=dev["o"], h0=dev["h0"])
    near(f64(y), S.scan(**val)[0], "bf16", "y")


def test_step_sizes_at_their_ends():
    """delta from far below zero, where D = exp(delta), to far above, where D =
    delta: D's relative error is that of a few roundings everywhere.  From the
    states: h = D b with a = 0 and x = 1."""
    torch, D = lib()
    F = 4096
    z = np.concatenate([np.linspace(-85, 85, F // 2), np.linspace(-4, 4, F // 2)])
    delta, dv = rounded(torch, z[None, None], "f32")
    one = torch.ones(1, 1, F, device="cuda")
    b = torch.ones(1, 1, 1, device="cuda")
    h, y = torch.empty(1, 1, F, device="cuda"), torch.empty(1, 1, F, device="cuda")
    D.dtst_scan(one, delta, torch.zeros(1, F, device="cuda"), b, b, y, h_out=h)
    off = np.abs(f64(h)[0, 0] / np.logaddexp(0.0, dv[0, 0]) - 1) * 2 ** 24
    say(f"[scan] D off by up to {off.max():.2f}, on average {off.mean():.2f} units of 2^-24")
    # exp 3 (its own 2, the argument's remainder 1), 1 + e 1, log 2, log 2 and the sum 1 each, the
    # first order 1
    assert off.max() <= 9


def test_infinite_states_and_no_numbers():
    """A state stays infinite while its decay is above zero, wherever segments
    begin; a no number stays in its feature."""
    torch, D = lib()
    T, F, N = 4000, 70, 2
    dev, val = inputs(torch, 1, T, F, N, "f32", 11, gated=False)
    dev["h0"] = dev["h0"].abs()
    dev["h0"][0, 0, 3] = float("inf")
    dev["a"][:, :] = -1.0
    dev["x"][0, 100, 5] = float("nan")
    y, h, _ = run(torch, D, dev, "f32")
    assert torch.isinf(h[0, 0, 3]) and torch.isfinite(h[0, 1, 3]) and torch.isinf(y[0, :, 3]).all()
    assert torch.isnan(h[0, :, 5]).all() and torch.isnan(y[0, 100:, 5]).all() and torch.isfinite(y[0, :100, 5]).all()
    ok = [i for i in range(F) if i not in (3, 5)]
    assert torch.isfinite(y[0][:, ok]).all()
    dev["a"][0, 3] = -1e4   # exp of it is below the smallest number: the state is gone, or no number
    _, h, _ = run(torch, D, dev, "f32")
    assert not torch.isinf(h[0, 0, 3])


@pytest.mark.parametrize("T", [48, 4000])
def test_step_sizes_whose_sums_pass_32_bits(T):
    """A state without decay stands still, and so does its gradient, however large the
    steps are: exact, as exp(0) is 1 and the others' 0."""
    torch, D = lib()
    F, N = 70, 2
    x, b = torch.zeros(1, T, F, device="cuda"), torch.zeros(1, T, N, device="cuda")
    c, delta = torch.ones(1, T, N, device="cuda"), torch.full((1, T, F), 3e38, device="cuda")
    a = torch.tensor([[0.0], [-1.0]], device="cuda").repeat(1, F)
    h, y = torch.ones(1, N, F, device="cuda"), torch.empty(1, T, F, device="cuda")
    st = torch.empty(D.scan_states_shape(1, T, F, N), device="cuda")
    D.dtst_scan(x, delta, a, b, c, y, h0=h, h_out=h, states=st)
    assert (y == 1).all() and (h[0, 0] == 1).all() and not h[0, 1].any()
    g_h, (g_b, g_c) = torch.ones_like(h), (torch.empty_like(b) for _ in range(2))
    g_x, g_delta = torch.empty_like(x), torch.empty_like(x)
    D.dtst_scan_adj(x, delta, a, b, c, torch.zeros_like(x), st, g_x, g_delta, torch.empty_like(a), g_b, g_c, g_h=g_h,
                    g_hzero=g_h)
    assert (g_h[0, 0] == 1).all() and not g_h[0, 1].any() and not g_x.any() and not g_delta.any() and not g_b.any()


def test_no_steps_and_no_sequences():
    torch, D = lib()
    dev, _ = inputs(torch, 2, 4, 10, 3, "f32", 12)
    e = {k: dev[k][:, :0] for k in ("x", "delta", "b", "c", "o")}
    h = empty(torch, "f32", 2, 3, 10)
    D.dtst_scan(e["x"], e["delta"], dev["a"], e["b"], e["c"], e["x"].clone(), o=e["o"], h0=dev["h0"], h_out=h)
    assert torch.equal(h, dev["h0"])
    D.dtst_scan(e["x"], e["delta"], dev["a"], e["b"], e["c"], e["x"].clone(), h_out=h)
    assert not h.any()
    n = {k: dev[k][:0] for k in ("x", "delta", "b", "c")}
    D.dtst_scan(n["x"], n["delta"], dev["a"], n["b"], n["c"], n["x"].clone())


def test_streams_and_graphs():
    """Two streams in turns, a workspace each; a graph replayed with eager work between."""
    torch, D = lib()
    dev, val = inputs(torch, 2, 700, 130, 5, "bf16", 13)
    want, h, _ = compare(torch, D, dev, val, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    ys = [empty(torch, "bf16", 2, 700, 130) for _ in range(8)]
    for i in range(0, 8, 2):
        for k, stream in enumerate((s.cuda_stream, None)):
            D.dtst_scan(dev["x"], dev["delta"], dev["a"], dev["b"], dev["c"], ys[i + k], d=dev["d"], o=dev["o"],
                        h0=dev["h0"], stream=stream)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys)
    state, y = dev["h0"].clone(), torch.empty_like(want)
    ws = torch.empty(D.dtst_scan_workspace(2, 700, 130, 5), dtype=torch.uint8, device="cuda")
    call = lambda y, st, w: D.dtst_scan(dev["x"], dev["delta"], dev["a"], dev["b"], dev["c"], y, d=dev["d"], o=dev["o"],  # noqa: E731
                                        h0=st, h_out=st, ws=w)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        call(y, state, ws)
    other = dev["h0"].clone()
    for k in range(4):
        ws.fill_(255)
        y.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        again = torch.empty_like(y)
        call(again, other, None)
        assert torch.equal(y, again) and torch.equal(state, other)


def test_refusals():
    torch, D = lib()
    dev, _ = inputs(torch, 2, 6, 10, 3, "bf16", 14)
    y, h = torch.empty(2, 6, 10, dtype=torch.bfloat16, device="cuda"), dev["h0"]
    good = dict(x=dev["x"], delta=dev["delta"], a=dev["a"], b=dev["b"], c=dev["c"], y=y, d=dev["d"], o=dev["o"], h0=h, h_out=h)
    pos = ("x", "delta", "a", "b", "c", "y")

    def call(**kw):
        k = dict(good, **kw)
        args = [k.pop(p) for p in pos]
        D.dtst_scan(*args, **k)

    call()
    for bad in (dict(x=dev["x"].float()), dict(x=dev["x"][0]), dict(x=dev["x"].double()), dict(delta=dev["delta"][:, :5]),
                dict(a=dev["a"].half()), dict(a=dev["a"][:, :9]), dict(a=dev["a"][0]), dict(b=dev["b"][..., :2]),
                dict(c=dev["c"].cpu()), dict(y=y.float()), dict(y=y[..., :9]), dict(d=dev["d"][:9]), dict(d=dev["d"].half()),
                dict(o=dev["o"][:1]), dict(h0=h[:, :2]), dict(h_out=h.transpose(1, 2)), dict(h0=h.double()),
                dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")),
                dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(states=h),
                dict(x=dev["x"].transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(D.DtstError):
        call(y=dev["x"])
    with pytest.raises(D.DtstError):
        call(a=torch.zeros(65, 10, device="cuda"), b=torch.zeros(2, 6, 65, dtype=torch.bfloat16, device="cuda"),
             c=torch.zeros(2, 6, 65, dtype=torch.bfloat16, device="cuda"), h0=None, h_out=None)
