"""The gated linear recurrence and its backward against the fp64 oracle:
lengths of none, one and many steps, feature counts around the lanes, unlike
lengths with no numbers past them, column ranges, missing arguments, states in
place, gates at their ends, long strides, other streams, graph replays."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from seq_common import dtype, f64, near, outside, rounded

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


class Case:
    """Inputs on the device as column ranges of one array, and in 64 bits."""

    def __init__(self, torch, B, T, F, t, seed, lengths=None, pad=0, gated=True, start=True):
        rng = np.random.RandomState(seed)
        self.shape, self.t, self.lengths = (B, T, F), t, lengths
        p = np.concatenate([rng.randn(B, T, F) * 2 + 1.5, rng.randn(B, T, 2 * F)], axis=2)
        g = rng.randn(B, T, F)
        if lengths is not None:
            for b in range(B):
                p[b, max(0, lengths[b]):] = np.nan
                g[b, max(0, lengths[b]):] = np.nan
        pd, pv = rounded(torch, p, t)
        wide = torch.full((B, T, 3 * F + pad), float("nan"), device="cuda").to(pd.dtype)
        wide[..., pad:] = pd
        self.z, self.v, self.o = (wide[..., pad + i * F:pad + (i + 1) * F] for i in range(3))
        self.zv, self.vv, self.ov = pv[..., :F], pv[..., F:2 * F], pv[..., 2 * F:]
        if not gated:
            self.o = self.ov = None
        self.h0, self.h0v = rounded(torch, rng.randn(B, F), "f32") if start else (None, None)
        self.g, self.gv = rounded(torch, g, t)
        self.gh, self.ghv = rounded(torch, rng.randn(B, F), "f32") if start else (None, None)
        self.n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        self.wide = torch.full((B, T, 3 * F + pad), float("nan"), device="cuda").to(pd.dtype)
        self.pad = pad


def run(torch, D, c, adj=True):
    B, T, F = c.shape
    e = dtype(torch, c.t)
    y = torch.full((B, T, F), float("nan"), device="cuda").to(e)
    h = torch.full((B, F), float("nan"), device="cuda")
    st = torch.full(D.recurrence_states_shape(B, T, F), float("nan"), device="cuda")
    D.dtst_recurrence(c.z, c.v, y, o=c.o, h0=c.h0, h_out=h, lengths=c.n, states=st)
    ry, rh = S.recurrence(c.zv, c.vv, c.ov, c.h0v, c.lengths)
    one = max(1.0, float(np.sqrt((rh ** 2).mean())))
    near(f64(y), ry, c.t, "y", rms=one)
    near(f64(h), rh[:, -1], "f32", "h", rms=one)
    near(f64(st), rh[:, 0:T:D.RECURRENCE_SPAN], "f32", "states", rms=one)
    if not adj:
        return y, h
    o = c.pad
    g_z, g_v, g_o = (c.wide[..., o + i * F:o + (i + 1) * F] for i in range(3))
    g0 = torch.full((B, F), float("nan"), device="cuda")
    D.dtst_recurrence_adj(c.z, c.v, c.g, st, g_z, g_v, o=c.o, g_o=g_o if c.o is not None else None, g_h=c.gh,
                          g_hzero=g0, lengths=c.n)
    rz, rv, ro, r0 = S.recurrence_adj(c.zv, c.vv, c.gv, rh, c.ov, c.ghv, c.lengths)
    # d sums up to 1 / (1 - s) terms: the bar is relative to its size
    size = max(1.0, *(float(np.abs(a).max()) for a in (rz, rv, ro, r0) if a.size))
    near(f64(g_z), rz, c.t, "g_z", rms=size)
    near(f64(g_v), rv, c.t, "g_v", rms=size)
    if c.o is not None:
        near(f64(g_o), ro, c.t, "g_o", rms=size)
    near(f64(g0), r0, "f32", "g_hzero", rms=size)
    if c.pad:
        assert bool(torch.isnan(c.wide[..., :c.pad].float()).all())
    return y, h


STEPS = [0, 1, 2, 7, 8, 9, 31, 32, 33, 64, 100, 127, 128, 129, 200, 255, 256, 257, 300, 511, 513, 1000, 1025, 2500]


@pytest.mark.parametrize("T", STEPS)
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_steps(T, t):
    torch, D = lib()
    say(f"[recurrence] 2 x {T} x 130 {t}")
    run(torch, D, Case(torch, 2, T, 130, t, T))


@pytest.mark.parametrize("F", [1, 2, 3, 63, 64, 65, 126, 127, 128, 129, 256, 257, 511, 1001])
@pytest.mark.parametrize("T", [1, 140, 600])
def test_features(F, T):
    torch, D = lib()
    say(f"[recurrence] 3 x {T} x {F}")
    run(torch, D, Case(torch, 3, T, F, "bf16", F, pad=F % 5))
    run(torch, D, Case(torch, 1, T, F, "f32", F + 1, gated=False))


@pytest.mark.parametrize("T", [1, 5, 130, 700, 1500])
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_unlike_lengths(T, t):
    torch, D = lib()
    n = [0, 1, T, max(0, T - 1), T // 2, -3 if T > 5 else 0, min(T, 128), min(T, 257)]
    say(f"[recurrence] lengths {n} of {T} {t}")
    run(torch, D, Case(torch, len(n), T, 67, t, T, lengths=n))


def test_lengths_past_the_end_mean_all():
    torch, D = lib()
    c = Case(torch, 2, 150, 40, "f32", 3)
    a, _ = run(torch, D, c)
    c.lengths, c.n = [150, 150], torch.tensor([1 << 30, 151], dtype=torch.int32, device="cuda")
    b, _ = run(torch, D, c)
    assert torch.equal(a, b)


@pytest.mark.parametrize("T", [1, 300])
def test_without_the_optional_arrays(T):
    torch, D = lib()
    c = Case(torch, 2, T, 70, "bf16", 5, gated=False, start=False)
    run(torch, D, c)
    y = torch.empty((2, T, 70), dtype=torch.bfloat16, device="cuda")
    D.dtst_recurrence(c.z, c.v, y)
    near(f64(y), S.recurrence(c.zv, c.vv)[0], "bf16", "y")


def test_serving_steps_in_place_follow_the_whole_sequence():
    torch, D = lib()
    c = Case(torch, 5, 20, 333, "bf16", 6)
    y, h = run(torch, D, c, adj=False)
    state = c.h0.clone()
    out = torch.empty_like(y)
    for t in range(20):
        D.dtst_recurrence(c.z[:, t:t + 1], c.v[:, t:t + 1], out[:, t:t + 1], o=c.o[:, t:t + 1], h0=state, h_out=state)
    near(f64(state), f64(h), "f32", "state")
    near(f64(out), f64(y), "bf16", "outputs")
    # the gradient's in place too
    st = torch.empty(D.recurrence_states_shape(*c.shape), device="cuda")
    D.dtst_recurrence(c.z, c.v, y, o=c.o, h0=c.h0, states=st)
    g = [torch.empty_like(y) for _ in range(6)]
    g0 = torch.empty_like(c.gh)
    D.dtst_recurrence_adj(c.z, c.v, c.g, st, g[0], g[1], o=c.o, g_o=g[2], g_h=c.gh, g_hzero=g0)
    D.dtst_recurrence_adj(c.z, c.v, c.g, st, g[3], g[4], o=c.o, g_o=g[5], g_h=c.gh, g_hzero=c.gh)
    assert torch.equal(g0, c.gh) and all(torch.equal(g[i], g[i + 3]) for i in range(3))


def test_gates_at_their_ends():
    torch, D = lib()
    T, F = 400, 8
    c = Case(torch, 1, T, F, "f32", 7)
    for i, v in enumerate((np.inf, -np.inf, 200.0, -200.0, 88.8, -88.8, 1e30, -1e30)):
        c.z[..., i] = v
        c.zv[..., i] = np.float32(v)
    c.o[0, :8, 0] = torch.tensor([200.0, -200.0, 88.8, -88.8, 0.0, -0.0, 3e38, -3e38])
    c.ov[0, :8, 0] = c.o[0, :8, 0].cpu().double().numpy()
    c.gv[0, 6] = c.g[0, 6] = 0      # (3e38 times a gradient of one passes fp32)
    y = torch.empty((1, T, F), device="cuda")
    h = torch.empty((1, F), device="cuda")
    D.dtst_recurrence(c.z, c.v, y, o=c.o, h0=c.h0, h_out=h)
    ry, rh = S.recurrence(c.zv, c.vv, c.ov, c.h0v)
    got, ref = f64(y), ry
    ok = np.abs(ref) < 1e30
    near(got[ok], ref[ok], "f32", "y")
    near(f64(h), rh[:, -1], "f32", "h")
    assert torch.equal(h[0, 0], c.h0[0, 0])         # an open gate keeps the state


def test_no_numbers_stay_in_their_feature_and_after_their_step():
    torch, D = lib()
    c = Case(torch, 2, 700, 66, "f32", 8)
    c.v[1, 300, 9] = float("nan")
    y = torch.empty((2, 700, 66), device="cuda")
    D.dtst_recurrence(c.z, c.v, y, o=c.o, h0=c.h0)
    bad = torch.isnan(y)
    assert bad[1, 300:, 9].all() and int(bad.sum()) == 400


def test_rows_past_32_bits():
    torch, D = lib()
    B, T, F = 2, 300, 70
    c = Case(torch, B, T, F, "bf16", 10)
    big = torch.empty((T, 1 << 24), dtype=torch.bfloat16, device="cuda")     # steps 2^24 apart: over 2^32 elements
    views = [big.as_strided((B, T, F), (4096, 1 << 24, 1), 1 + 128 * i) for i in range(8)]
    for src, dst in zip((c.z, c.v, c.o, c.g), views):
        dst.copy_(src)
    st = torch.empty(D.recurrence_states_shape(B, T, F), device="cuda")
    D.dtst_recurrence(views[0], views[1], views[4], o=views[2], h0=c.h0, states=st)
    ry, rh = S.recurrence(c.zv, c.vv, c.ov, c.h0v)
    near(f64(views[4]), ry, "bf16", "y")
    D.dtst_recurrence_adj(views[0], views[1], views[3], st, views[5], views[6], o=views[2], g_o=views[7], g_h=c.gh)
    want = S.recurrence_adj(c.zv, c.vv, c.gv, rh, c.ov, c.ghv)
    for got, ref, name in zip(views[5:], want, ("g_z", "g_v", "g_o")):
        near(f64(got), ref, "bf16", name)


def test_another_stream():
    torch, D = lib()
    c = Case(torch, 2, 3000, 200, "bf16", 11)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y1, y2 = (torch.empty((2, 3000, 200), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for _ in range(4):
        D.dtst_recurrence(c.z, c.v, y1, o=c.o, h0=c.h0, stream=s.cuda_stream)   # workspace of the call itself
        D.dtst_recurrence(c.z, c.v, y2, o=c.o, h0=c.h0)
    torch.cuda.synchronize()
    assert torch.equal(y1, y2)
    near(f64(y1), S.recurrence(c.zv, c.vv, c.ov, c.h0v)[0], "bf16", "y")


def test_graph_replays():
    torch, D = lib()
    c = Case(torch, 2, 2000, 130, "bf16", 12)
    B, T, F = c.shape
    y, h = torch.empty_like(c.g), torch.empty_like(c.h0)
    st = torch.empty(D.recurrence_states_shape(B, T, F), device="cuda")
    g = [torch.empty_like(c.g) for _ in range(3)]
    n = D.dtst_recurrence_workspace(B, T, F, torch.bfloat16)
    ws = torch.empty(max(16, n), dtype=torch.uint8, device="cuda")

    def step():
        D.dtst_recurrence(c.z, c.v, y, o=c.o, h0=c.h0, h_out=h, states=st, ws=ws)
        D.dtst_recurrence_adj(c.z, c.v, c.g, st, g[0], g[1], o=c.o, g_o=g[2], g_h=c.gh, ws=ws)

    step()
    want = [a.clone() for a in (y, h, *g)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for a in (y, h, st, ws, *g):
            a.view(torch.uint8).fill_(i + 1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (y, h, *g))), i


@pytest.mark.parametrize("B,T,F", [(4096, 1, 129), (512, 1, 1025), (96, 300, 257), (40, 128, 641)])
def test_states_in_place_where_a_feature_is_left_over(B, T, F):
    """A last tile of a single feature shares none with the one before."""
    torch, D = lib()
    c = Case(torch, B, T, F, "bf16", F)
    y, h, st = torch.empty_like(c.g), c.h0.clone(), torch.empty(D.recurrence_states_shape(B, T, F), device="cuda")
    y2, h2 = torch.empty_like(c.g), torch.empty_like(c.h0)
    D.dtst_recurrence(c.z, c.v, y, o=c.o, h0=h, h_out=h, states=st)
    D.dtst_recurrence(c.z, c.v, y2, o=c.o, h0=c.h0, h_out=h2)
    assert torch.equal(h, h2) and torch.equal(y, y2)
    g = [torch.empty_like(c.g) for _ in range(3)]
    gh, gh2 = c.gh.clone(), torch.empty_like(c.gh)
    D.dtst_recurrence_adj(c.z, c.v, c.g, st, g[0], g[1], o=c.o, g_o=g[2], g_h=gh, g_hzero=gh)
    D.dtst_recurrence_adj(c.z, c.v, c.g, st, g[0], g[1], o=c.o, g_o=g[2], g_h=c.gh, g_hzero=gh2)
    assert torch.equal(gh, gh2)
    near(f64(h2), S.recurrence(c.zv, c.vv, c.ov, c.h0v)[1][:, -1], "f32", "h",
         rms=max(1.0, float(np.abs(c.h0v).max())))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("B,T,F", [(130, 1, 2), (130, 17, 3), (150, 16, 127), (70, 40, 130), (70, 128, 254),
                                   (66, 129, 200), (45, 300, 127), (6, 3300, 2), (33, 257, 386), (129, 1, 128)])
def test_many_workgroups(B, T, F, t):
    """Enough of them that a lane takes two features."""
    torch, D = lib()
    run(torch, D, Case(torch, B, T, F, t, B + T + F))


@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_many_workgroups_of_unlike_lengths(t):
    torch, D = lib()
    B, T = 48, 390
    lengths = [0, 1, 15, 16, 17, 127, 128, 129, 200, 255, 256, 257, 383, 384, 385, 389, 390, 400, -3] * 3
    run(torch, D, Case(torch, B, T, 131, t, 5, lengths=lengths[:B], pad=3))
