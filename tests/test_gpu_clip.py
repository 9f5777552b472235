"""The norm of many tensors together and their scaling against 64 bits: counts
around the chunks' limits, more tensors than a launch takes, mixed and complex
types, odd addresses, values whose squares pass 32 bits, no numbers and
infinities, graphs."""

import math

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from seq_common import HALF_STEP, LEAST, dtype, f64, rounded

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def norm64(ts):
    return math.sqrt(math.fsum(float((f64(t) ** 2).sum()) for t in ts))


def check(torch, D, ts, most, in_place=False, norm=None):
    n = torch.empty((), device="cuda")
    want = norm64(ts)
    D.dtst_global_norm(ts, n)
    # 64-bit sums (count 2^-53 at most), then one rounding
    assert abs(float(n) - want) <= 2.0 ** -23 * want, (float(n), want)
    before = [f64(t) for t in ts]
    out = None if in_place else [torch.full_like(t, 7.0) for t in ts]
    D.dtst_clip(ts, n, most, out=out)
    f = 1.0 if want <= most else most / want
    for i, (b, o, t) in enumerate(zip(before, ts if in_place else out, ts)):
        kind = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}[t.dtype]
        # the norm's, the quotient's and the product's rounding, and the type's own
        off = np.abs(f64(o) - b * f) - (HALF_STEP[kind] + 4 * 2.0 ** -24) * np.abs(b * f) - LEAST[kind]
        assert b.size == 0 or off.max() <= 0, (i, kind, off.max())
        if not in_place:
            assert np.array_equal(f64(t), b)


def make(torch, counts, kinds, seed, std=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(n, generator=g, device="cuda") * std).to(dtype(torch, kinds[i % len(kinds)]))
            for i, n in enumerate(counts)]


@pytest.mark.parametrize("kinds", [("f32",), ("bf16",), ("f16",), ("f32", "bf16", "f16")])
@pytest.mark.parametrize("counts", [(1,), (0,), (0, 5, 0), (8191, 8192, 8193), (3, 100000, 1, 0, 77, 8192 * 5),
                                    (8192 * 2100 + 3, 9)], ids=str)
@pytest.mark.parametrize("in_place", [False, True])
def test_counts(kinds, counts, in_place):
    torch, D = lib()
    say(f"[clip] {counts} {kinds}")
    ts = make(torch, counts, kinds, sum(counts))
    check(torch, D, ts, 0.5 * norm64(ts), in_place)
    check(torch, D, ts, 2.0 * norm64(ts) + 1, in_place)   # nothing to scale


@pytest.mark.parametrize("n", [127, 128, 129, 183, 184, 185, 700])
def test_many_tensors(n):
    torch, D = lib()
    rng = np.random.RandomState(n)
    ts = make(torch, rng.randint(0, 12000, n), ("f32", "bf16"), n)
    check(torch, D, ts, 3.0)
    check(torch, D, ts, 2.0, in_place=True)


def test_no_tensors():
    torch, D = lib()
    n = torch.full((1,), 5.0, device="cuda")
    D.dtst_global_norm([], n)
    assert float(n) == 0
    D.dtst_clip([], n, 1.0)
    D.dtst_clip([], n, 1.0, out=[])


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_neighbours_at_odd_addresses(kind):
    """Runs of one array, one after the other, between guards."""
    torch, D = lib()
    counts = [1, 2, 8190, 3, 20001, 5]
    a, b = torch.randn(sum(counts) + 2, device="cuda").to(dtype(torch, kind)), torch.empty(0)
    b = torch.full_like(a, 9.0)
    ts, outs = a[1:-1].split(counts), b[1:-1].split(counts)
    n = torch.empty(1, device="cuda")
    D.dtst_global_norm(ts, n)
    want = norm64(ts)
    assert abs(float(n) - want) <= 2.0 ** -23 * want
    D.dtst_clip(ts, n, 1.0, out=outs)
    assert float(b[0]) == 9 and float(b[-1]) == 9
    ref = f64(a)[1:-1] / want
    assert (np.abs(f64(b)[1:-1] - ref) <= (HALF_STEP[kind] + 2.0 ** -22) * np.abs(ref)).all()


def test_complex_gradients():
    torch, D = lib()
    w = torch.randn(50, 3, 4, dtype=torch.complex64, device="cuda")
    b = torch.randn(7, device="cuda")
    n, out = torch.empty(1, device="cuda"), [torch.empty_like(w), torch.empty_like(b)]
    D.dtst_global_norm([w, b], n)
    want = math.sqrt(norm64([torch.view_as_real(w)]) ** 2 + norm64([b]) ** 2)
    assert abs(float(n) - want) <= 2.0 ** -23 * want
    D.dtst_clip([w, b], n, 0.25, out=out)
    assert torch.allclose(out[0], w * (0.25 / want), rtol=1e-6, atol=0) and torch.allclose(out[1], b * (0.25 / want), rtol=1e-6, atol=0)
    with pytest.raises(ValueError):
        D.dtst_global_norm([w.conj()], n)


def test_values_whose_squares_pass_32_bits():
    torch, D = lib()
    for std in (1e30, 1e-30):
        ts = make(torch, (1000, 9000), ("f32",), 1, std)
        check(torch, D, ts, 0.3 * norm64(ts))
    n = torch.empty(1, device="cuda")
    D.dtst_global_norm([torch.full((1 << 16,), 3e38, device="cuda")], n)   # beyond 32 bits
    assert math.isinf(float(n))


# Eight values whose squares, added one after the other in 32 bits, put the norm 2.7, 3.1
# and 2.7 units of 2^-24 off.
EIGHT = {
    "f32": ["0x1.04e430p-1", "0x1.6ddcd0p+0", "0x1.59e5d0p-1", "0x1.1b8b80p-1", "0x1.0e5008p+0", "0x1.c9a3d4p-2",
            "0x1.1213f8p-2", "0x1.7ee75ap-3"],
    "bf16": [0.0308837890625, 0.53125, 0.0257568359375, 0.0252685546875, 0.0308837890625, 0.036865234375, 0.0294189453125,
             0.013916015625],
    "f16": [0.744140625, 0.89111328125, 0.94140625, 1.4384765625, 0.30615234375, 0.44189453125, 0.66845703125, 0.25537109375],
}


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_norm_of_one_group_and_of_equal_values(kind):
    """The root's rounding to 32 bits, 2^-24, and half of those of two neighbours' squares:
    two of 2^-24 of their sum (the first square's and the sum's), one of a 16-bit type,
    whose squares 32 bits hold.  One group of eight, whose own roundings are all there
    are, and equal values, whose roundings are all alike."""
    torch, D = lib()
    rng = np.random.RandomState(3)
    bar = 2.0 if kind == "f32" else 1.5
    values = [[float.fromhex(v) if isinstance(v, str) else v for v in EIGHT[kind]]]
    values += list(rng.uniform(1, 2, (100, 8))) + [np.full(65536 + 8 * i, v) for i, v in enumerate(rng.uniform(1, 2, 100))]
    values.append(np.full(65536, float.fromhex("0x1.cca210p+0")))
    ts = [rounded(torch, v, kind)[0] for v in values]
    n = torch.empty(len(ts), device="cuda")
    for i, t in enumerate(ts):
        D.dtst_global_norm([t], n[i])
    want = np.array([norm64([t]) for t in ts])
    off = np.abs(f64(n) / want - 1) * 2 ** 24
    say(f"[clip] {kind}: the norm of eight {off[0]:.3f}, of others up to {off[1:101].max():.3f}, of equal ones up to "
        f"{off[101:].max():.3f} units of 2^-24 off")
    assert off.max() <= bar * (1 + 1e-6)


def test_no_numbers_and_infinities():
    torch, D = lib()
    n = torch.empty(1, device="cuda")
    a, b = torch.ones(9, device="cuda"), torch.ones(5, device="cuda", dtype=torch.bfloat16)
    a[3] = float("inf")
    outs = [torch.empty_like(a), torch.empty_like(b)]
    D.dtst_global_norm([a, b], n)
    D.dtst_clip([a, b], n, 1.0, out=outs)
    assert math.isinf(float(n)) and not outs[1].any() and torch.isnan(outs[0][3]) and not outs[0][:3].any()
    D.dtst_clip([a, b], n, float("inf"), out=outs)
    assert torch.equal(outs[0], a) and torch.equal(outs[1], b)
    a[3] = float("nan")
    D.dtst_global_norm([a, b], n)
    D.dtst_clip([a, b], n, 1.0, out=outs)
    assert math.isnan(float(n)) and torch.isnan(outs[0]).all() and torch.isnan(outs[1].float()).all()
    z = [torch.zeros(30, device="cuda")]
    D.dtst_global_norm(z, n)
    D.dtst_clip(z, n, 0.0)
    assert float(n) == 0 and not z[0].any()
    z = [torch.ones(30, device="cuda")]
    D.dtst_global_norm(z, n)
    D.dtst_clip(z, n, 0.0)
    assert not z[0].any()


def test_repeated_and_replayed():
    """The same bits every time, in a graph too, with eager work between the replays."""
    torch, D = lib()
    ts = make(torch, (100000, 17, 0, 8192 * 3), ("f32", "bf16"), 5)
    n, want, outs = torch.empty(1, device="cuda"), torch.empty(1, device="cuda"), [torch.empty_like(t) for t in ts]
    D.dtst_global_norm(ts, want)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        D.dtst_global_norm(ts, n, ws=ws)
        D.dtst_clip(ts, n, 1.0, out=outs)
    for k in range(4):
        for t in ts:
            t.mul_(0.5)
        ws.fill_(255)
        n.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        D.dtst_global_norm(ts, want)
        assert torch.equal(n, want)
        eager = [torch.empty_like(t) for t in ts]
        D.dtst_clip(ts, want, 1.0, out=eager)
        assert all(torch.equal(a, b) for a, b in zip(outs, eager))


def test_refusals():
    torch, D = lib()
    a, n = torch.ones(100, device="cuda"), torch.empty(1, device="cuda")
    for bad in ([a.double()], [a.cpu()], [a[::2]], [a, a.view(10, 10).t()], [a.to(torch.float8_e4m3fn)]):
        with pytest.raises(ValueError):
            D.dtst_global_norm(bad, n)
        with pytest.raises(ValueError):
            D.dtst_clip(bad, n, 1.0)
        with pytest.raises(ValueError):
            D.dtst_clip([a] * len(bad), n, 1.0, out=bad)
    for bad in (n.double(), n.cpu(), torch.empty(2, device="cuda")):
        with pytest.raises(ValueError):
            D.dtst_global_norm([a], bad)
        with pytest.raises(ValueError):
            D.dtst_clip([a], bad, 1.0)
    for out in ([a[:50]], [a, a], [a.half()]):
        with pytest.raises(ValueError):
            D.dtst_clip([a], n, 1.0, out=out)
    for bad in (lambda: D.dtst_clip([a], n, -1.0), lambda: D.dtst_clip([a], n, float("nan")),
                lambda: D.dtst_clip([a, a], n, 1.0), lambda: D.dtst_clip([a[:60], a[50:]], n, 1.0),
                lambda: D.dtst_clip([a[:50]], n, 1.0, out=[a[1:51]]), lambda: D.dtst_clip([a], a[5:6], 1.0),
                lambda: D.dtst_global_norm([a], a[7:8]), lambda: D.dtst_global_norm([a], n, ws=a[:1].view(torch.uint8)),
                lambda: D.dtst_global_norm([a], n, ws=a.view(torch.uint8))):
        with pytest.raises(D.DtstError):
            bad()
    D.dtst_global_norm([a, a[:50]], n)   # (counted twice)
    assert abs(float(n) - 150 ** 0.5) < 1e-5
    D.dtst_clip([a[:50], a[50:]], n, 1.0)
