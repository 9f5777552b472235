"""The latent-sequence operators together: a residual block's forward and
backward against their fp64 composition, sequences against serving steps, a
replayed serving step, and fields marched through a plan's coefficients."""

import numpy as np
import pytest

import oracle as O
from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from seq_common import f64, rounded

pytestmark = pytest.mark.gpu

# Between the operators results are rounded to bf16 (half a step 2^-8) and to
# e4m3 (2^-4); where the fp32 path and the oracle round to different neighbours
# a value differs by a whole step, rarely.  One bf16 step bounds the rest.
BAR = 2.0 ** -7


def rel(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


def bf16(torch, a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(torch.bfloat16).double().numpy()


def val(a):
    return S.values(*S.quantise(a))


class Block:
    """A block and its weights in 64 bits."""

    def __init__(self, torch, W, F, seed):
        from paper_2607_14394_amd.rollout import LatentBlock
        rng = np.random.RandomState(seed)
        self.W, self.F = W, F
        self.norm_d, self.norm = rounded(torch, 1 + 0.2 * rng.randn(W), "f32")
        self.w_in_d, self.w_in = rounded(torch, rng.randn(3 * F, W) / np.sqrt(W), "f32")
        self.b_d, self.b = rounded(torch, 0.5 * rng.randn(3 * F) + np.repeat([1.5, 0, 0], F), "f32")
        self.w_out_d, self.w_out = rounded(torch, rng.randn(W, F) / np.sqrt(F), "f32")
        self.block = LatentBlock(self.norm_d, self.w_in_d, self.b_d, self.w_out_d)


def forward64(torch, k, x, res, h0, lengths, plain_norm):
    """The composition, rounded where the operators' types round."""
    B, T, W = x.shape
    u = np.float32(x) + np.float32(res)
    u = u.astype(np.float64)
    n, rstd = S.rms_norm(u.reshape(-1, W), k.norm, 1e-6)
    n = val(bf16(torch, n) if plain_norm else n)[:, :W]
    p = bf16(torch, S.product(n, val(k.w_in)[:, :W], k.b)).reshape(B, T, 3 * k.F)
    z, v, o = p[..., :k.F], p[..., k.F:2 * k.F], p[..., 2 * k.F:]
    y, h = S.recurrence(z, v, o, h0, lengths)
    y = bf16(torch, y)
    out = S.product(val(y.reshape(-1, k.F))[:, :k.F], val(k.w_out)[:, :k.F]).reshape(B, T, W)
    return dict(u=u, p=p, y=y, h=h, out=out, n=n)


@pytest.mark.parametrize("B,T,W,F,lengths", [(2, 5, 200, 96, None), (3, 300, 384, 130, [300, 0, 171]), (1, 1, 640, 256, None)])
def test_block_forward_and_backward(B, T, W, F, lengths):
    torch = torch_gpu()
    k = Block(torch, W, F, T)
    rng = np.random.RandomState(W)
    x, xv = rounded(torch, rng.randn(B, T, W), "bf16")
    res, rv = rounded(torch, 2 * rng.randn(B, T, W), "f32")
    h0, hv = rounded(torch, rng.randn(B, F), "f32")
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    say(f"[block] {B} x {T} x {W}, {F} features, lengths {lengths}")
    state, keep = h0.clone(), {}
    out, u = k.block.forward(x, res, state, n, keep)
    r = forward64(torch, k, xv, rv, hv, lengths, plain_norm=True)
    assert np.array_equal(f64(u), r["u"]) and np.array_equal(f64(res), rv)
    for name, got, ref in (("branch", f64(out), r["out"]), ("state", f64(state), r["h"][:, -1])):
        say(f"  {name}: rel {rel(got, ref):.2e}")
        assert rel(got, ref) <= BAR, name
    # serving form: the norm straight to 8 bits, the residual in place
    state2, res2 = h0.clone(), res.clone()
    out2, u2 = k.block.forward(x, res2, state2, n)
    r2 = forward64(torch, k, xv, rv, hv, lengths, plain_norm=False)
    assert u2.data_ptr() == res2.data_ptr() and np.array_equal(f64(res2), r["u"])
    assert rel(f64(out2), r2["out"]) <= BAR and rel(f64(state2), r2["h"][:, -1]) <= BAR

    g_out, gov = rounded(torch, rng.randn(B, T, W), "bf16")
    g_res, grv = rounded(torch, rng.randn(B, T, W), "f32")
    g_h, ghv = rounded(torch, rng.randn(B, F), "f32")
    got = k.block.backward(keep, g_out, g_res, g_h)
    go = gov.reshape(-1, W)
    g_y = bf16(torch, S.product(val(go)[:, :W], val(k.w_out.T)[:, :W])).reshape(B, T, F)
    z, v, o = r["p"][..., :F], r["p"][..., F:2 * F], r["p"][..., 2 * F:]
    gz, gv, gg, g0 = S.recurrence_adj(z, v, g_y, r["h"], o, ghv, lengths)
    g_p = bf16(torch, np.concatenate([gz, gv, gg], axis=2)).reshape(-1, 3 * F)
    g_n = bf16(torch, S.product(val(g_p)[:, :3 * F], val(k.w_in.T)[:, :3 * F]))
    n_plain = bf16(torch, S.rms_norm(r["u"].reshape(-1, W), k.norm, 1e-6)[0])
    g_u, g_norm = S.rms_norm_adj(g_n, r["u"].reshape(-1, W), k.norm, 1e-6, grv.reshape(-1, W))
    R = B * T
    want = dict(x=g_u.reshape(B, T, W), res=g_u.reshape(B, T, W), state=g0, norm=g_norm,
                w_in=S.product(val(g_p.T)[:, :R], val(n_plain.T)[:, :R]), b_in=g_p.sum(axis=0),
                w_out=S.product(val(go.T)[:, :R], val(r["y"].reshape(-1, F).T)[:, :R]))
    for name, ref in want.items():
        e = rel(f64(got[name]), ref)
        say(f"  g_{name}: rel {e:.2e}")
        assert e <= BAR, name


def test_gradients_are_those_of_the_layer_without_8_bits():
    """Against autograd in 64 bits on unquantised weights: e4m3 keeps a value
    within 2^-4 of itself (2.6% rms), three products in a row within 20%."""
    torch = torch_gpu()
    B, T, W, F = 2, 40, 256, 128
    k = Block(torch, W, F, 3)
    rng = np.random.RandomState(4)
    x, xv = rounded(torch, rng.randn(B, T, W), "bf16")
    res, rv = rounded(torch, rng.randn(B, T, W), "f32")
    g, gv = rounded(torch, rng.randn(B, T, W), "bf16")
    t = {n: torch.tensor(a, requires_grad=True) for n, a in
         (("x", xv), ("norm", k.norm), ("w_in", k.w_in), ("b_in", k.b), ("w_out", k.w_out))}
    u = t["x"] + torch.tensor(rv)
    n = u / torch.sqrt((u * u).mean(dim=2, keepdim=True) + 1e-6) * t["norm"]
    z, v, o = (n @ t["w_in"].T + t["b_in"]).split(F, dim=2)
    h, ys = torch.zeros(B, F, dtype=torch.float64), []
    for i in range(T):
        s = torch.sigmoid(z[:, i])
        h = s * h + (1 - s) * v[:, i]
        ys.append(h * o[:, i] * torch.sigmoid(o[:, i]))
    out = torch.stack(ys, dim=1) @ t["w_out"].T
    out.backward(torch.tensor(gv))
    keep = {}
    got_out, _ = k.block.forward(x, res, keep=keep)
    got = k.block.backward(keep, g, None)
    assert rel(f64(got_out), out.detach().numpy()) <= 0.2
    for name, p in t.items():
        e = rel(f64(got[name]), p.grad.numpy())
        say(f"  g_{name}: rel {e:.2e}")
        assert e <= 0.2, name


def test_steps_follow_the_sequence_and_replay():
    torch = torch_gpu()
    B, T, W, F = 4, 12, 512, 320
    k = Block(torch, W, F, 7)
    rng = np.random.RandomState(8)
    x, _ = rounded(torch, rng.randn(B, T, W), "bf16")
    res, _ = rounded(torch, rng.randn(B, T, W), "f32")
    h0, _ = rounded(torch, rng.randn(B, F), "f32")
    state = h0.clone()
    out, u = k.block.forward(x, res.clone(), state)
    step_state, outs = h0.clone(), []
    for t in range(T):
        c, r = k.block.forward(x[:, t:t + 1].contiguous(), res[:, t:t + 1].contiguous(), step_state)
        outs.append(c)
        assert torch.equal(r[:, 0], u[:, t])
    assert rel(f64(torch.cat(outs, dim=1)), f64(out)) <= BAR and rel(f64(step_state), f64(state)) <= BAR
    # a serving step in a graph: its state goes on from replay to replay
    xs, rs, live = x[:, :1].contiguous(), res[:, :1].contiguous(), h0.clone()
    k.block.forward(xs, rs.clone(), h0.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c, _ = k.block.forward(xs, rs, live)
    live.copy_(h0)
    for t in range(T):
        xs.copy_(x[:, t:t + 1])
        rs.copy_(res[:, t:t + 1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(c, outs[t]), t
    assert torch.equal(live, step_state)


def test_fields_are_marched():
    torch = torch_gpu()
    from paper_2607_14394_amd.rollout import Rollout
    grid = dict(n_global=(16, 12, 20), n_local=(16, 12, 20), offset=(0, 0, 0), kmax=(2, 3, 2))
    B, T, C = 2, 6, 3
    W = 2 * C * 4 * 6 * 4
    blocks = [Block(torch, W, 192, s).block for s in (1, 2)]
    ro = Rollout(grid, C, B, blocks)
    assert ro.width == W
    rng = np.random.RandomState(5)
    f, fv = rounded(torch, rng.randn(B, T, C, 16, 12, 20), "f32")
    tok = ro.encode(f)
    g = O.Geometry((16, 12, 20, 1), (16, 12, 20, 1), (0, 0, 0, 0), (2, 3, 2), 1, B * T, C, C)
    ref = O.forward(fv.reshape(B * T, C, 16, 12, 20, 1), g)
    got = f64(tok).reshape(-1, 2)
    assert rel(got[:, 0] + 1j * got[:, 1], ref.ravel()) <= 1e-5
    back = f64(ro.decode(tok)).reshape(B * T, C, 16, 12, 20, 1)
    assert rel(back, O.inverse(ref, g)) <= 1e-5
    whole = ro.advance(f)
    ro.reset()
    steps = torch.cat([ro.advance(f[:, t:t + 1]) for t in range(T)], dim=1)
    say(f"  steps against the sequence: rel {rel(f64(steps), f64(whole)):.2e}")
    assert rel(f64(steps), f64(whole)) <= BAR
    far = ro.march(f[:, -1], 3)
    assert far.shape == (B, 3, C, 16, 12, 20) and bool(torch.isfinite(far).all())
    ro.close()


@pytest.mark.parametrize("B,T,C", [(1, 1, 3), (2, 131, 1), (1, 257, 2), (3, 67, 16)])
def test_more_frames_than_one_plan_takes(B, T, C):
    """Frames are encoded and decoded in groups: each frame as by itself."""
    torch = torch_gpu()
    from paper_2607_14394_amd.rollout import Rollout
    grid = dict(n_global=(8, 6, 8), n_local=(8, 6, 8), offset=(0, 0, 0), kmax=(1, 1, 2))
    ro = Rollout(grid, C, B, [])
    g = O.Geometry((8, 6, 8, 1), (8, 6, 8, 1), (0, 0, 0, 0), (1, 1, 2), 1, B * T, C, C)
    f, fv = rounded(torch, np.random.RandomState(T).randn(B, T, C, 8, 6, 8), "f32")
    tok = ro.encode(f)
    assert tok.shape == (B, T, 2 * C * 2 * 2 * 4)
    ref = O.forward(fv.reshape(B * T, C, 8, 6, 8, 1), g)
    got = f64(tok).reshape(-1, 2)
    assert rel(got[:, 0] + 1j * got[:, 1], ref.ravel()) <= 1e-5
    assert rel(f64(ro.decode(tok)).reshape(B * T, C, 8, 6, 8, 1), O.inverse(ref, g)) <= 1e-5
    ro.close()


def test_blocks_refuse_other_shapes():
    torch = torch_gpu()
    from paper_2607_14394_amd.rollout import LatentBlock, Rollout
    one = lambda *s: torch.ones(s, device="cuda")  # noqa: E731
    with pytest.raises(ValueError):
        LatentBlock(one(64), one(95, 64), one(96), one(64, 32))
    b = LatentBlock(one(64), one(96, 64), one(96), one(64, 32))
    with pytest.raises(ValueError):
        Rollout(dict(n_global=(8, 8, 8), n_local=(8, 8, 8), offset=(0, 0, 0), kmax=(1, 1, 1)), 1, 1, [b])


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), 1e30])
def test_what_lies_past_a_length_reaches_no_gradient(junk):
    """Zeros there or anything else: the same gradients, bit for bit."""
    torch = torch_gpu()
    B, T, W, F, lengths = 3, 130, 200, 96, [130, 0, 71]
    k = Block(torch, W, F, 5)
    rng = np.random.RandomState(6)
    n = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    past = (torch.arange(T, device="cuda") >= n[:, None])[..., None]
    x, res, g_out, g_res = (rounded(torch, rng.randn(B, T, W), t)[0] for t in ("bf16", "f32", "bf16", "f32"))
    h0, g_h = (rounded(torch, rng.randn(B, F), "f32")[0] for _ in range(2))
    say(f"[past lengths] {junk}")
    runs = []
    for fill in (0.0, junk):
        state, keep = h0.clone(), {}
        out, u = k.block.forward(x.masked_fill(past, fill), res.masked_fill(past, fill), state, n, keep)
        g = k.block.backward(keep, g_out.masked_fill(past, fill), g_res.masked_fill(past, fill), g_h)
        g.update(out=out, last=state, u=u.masked_fill(past, 0), x=g["x"].masked_fill(past, 0),
                 res=g["res"].masked_fill(past, 0))
        runs.append(g)
    for name, ref in runs[0].items():
        assert torch.isfinite(ref).all(), name
        assert torch.equal(runs[1][name], ref), name


@pytest.mark.parametrize("B,T", [(2, 0), (0, 3)])
@pytest.mark.parametrize("with_lengths", [False, True])
def test_a_block_over_no_steps(B, T, with_lengths):
    """The state stands still, its gradient passes, the others are zero."""
    torch = torch_gpu()
    W, F = 200, 96
    k = Block(torch, W, F, 7)
    say(f"[no steps] {B} x {T}, lengths {with_lengths}")
    n = torch.zeros(B, dtype=torch.int32, device="cuda") if with_lengths else None
    x, res = torch.zeros(B, T, W, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, T, W, device="cuda")
    h0, g_h = torch.randn(B, F, device="cuda"), torch.randn(B, F, device="cuda")
    state, keep = h0.clone(), {}
    out, u = k.block.forward(x, res, state, n, keep)
    assert out.shape == u.shape == (B, T, W) and torch.equal(state, h0)
    assert k.block.forward(x, res, state, n)[0].shape == (B, T, W) and torch.equal(state, h0)  # (the serving form)
    g = k.block.backward(keep, torch.zeros_like(out), torch.zeros_like(u), g_h)
    assert torch.equal(g["state"], g_h) and g["x"].shape == g["res"].shape == (B, T, W)
    for name, shape in (("norm", (W,)), ("w_in", (3 * F, W)), ("b_in", (3 * F,)), ("w_out", (W, F))):
        assert g[name].shape == shape and not g[name].any(), name
