"""Products of 8-bit arrays with block scales against the fp64 oracle on the
values that codes and scales stand for: sizes around every tile's limits, one
row and one column, the summed axis from one to many blocks, types, bias,
accumulation, strides, scales far apart, and a linear layer's gradients."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from oracle import seq_oracle as S
from seq_common import HALF_STEP, dtype, f64, near, outside, rounded, strided

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def codes(torch, D, v):
    """Codes, scales and the values that they stand for, from the oracle."""
    q, e = S.quantise(v)
    cq = torch.from_numpy(q).float().to(torch.float8_e4m3fn).cuda()
    s = np.full((v.shape[0], D.scale_columns(v.shape[1])), 127, np.uint8)
    s[:, :e.shape[1]] = e + 127
    return cq, torch.from_numpy(s).cuda().view(torch.float8_e8m0fnu), S.values(q, e)


def operand(rng, r, k):
    return rng.randn(r, k) * np.exp2(rng.uniform(-4, 4, (r, 1))) * np.where(rng.rand(1, k) < 0.02, 30, 1)


# rows of a and b: one, around 16, 32, 64, 128 and 256, and several tiles
SIZES = [(1, 1, 128), (1, 100, 1000), (2, 64, 512), (3, 300, 640), (4, 4608, 256), (8, 129, 2048), (15, 17, 129),
         (16, 16, 1), (17, 65, 513), (31, 256, 1024), (33, 127, 384), (63, 255, 130), (64, 64, 4096), (65, 257, 200),
         (100, 1000, 1900), (127, 129, 1152), (128, 128, 128), (129, 513, 896), (200, 1, 700), (255, 300, 1024),
         (256, 256, 256), (257, 255, 520), (500, 700, 300), (513, 640, 128), (777, 1000, 1900), (1025, 1030, 512),
         (1300, 2100, 640), (2048, 2048, 1024), (3500, 3700, 256)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_product(m, n, k):
    torch, D = lib()
    rng = np.random.RandomState(m * 7 + n * 3 + k)
    a, sa, av = codes(torch, D, operand(rng, m, k))
    b, sb, bv = codes(torch, D, operand(rng, n, k))
    bias, biasv = rounded(torch, rng.randn(n), "f32")
    say(f"[product] {m} x {n} x {k}")
    ref = S.product(av, bv)
    # each result's terms: what an fp32 sum of them may be off by scales with their size
    size = np.sqrt((av ** 2).sum(axis=1)[:, None] * (bv ** 2).sum(axis=1)[None, :])
    for t in ("f32", "bf16", "f16"):
        c = torch.full((m, n), float("nan"), device="cuda").to(dtype(torch, t))
        sc = 2.0 ** -6 if t == "f16" else 1.0   # (in range of the type)
        s8 = sa if t != "f16" else (sa.view(torch.uint8) - 6).view(torch.float8_e8m0fnu)
        D.dtst_product(a, s8, b, sb, c)
        got = f64(c) / size
        near(got, ref * sc / size, t, t, rms=1.0)
    c = torch.empty((m, n), device="cuda")
    D.dtst_product(a, sa, b, sb, c, bias=bias)
    near((f64(c) - biasv) / size, ref / size, "f32", "bias", arithmetic=2e-5, rms=1.0)
    base, basev = rounded(torch, rng.randn(m, n), "f32")
    D.dtst_product(a, sa, b, sb, base, accumulate=True)
    near((f64(base) - basev) / size, ref / size, "f32", "accumulate", arithmetic=2e-5, rms=1.0)


# The 8-bit instruction's sum of eight neighbouring products keeps 13 bits below
# the largest: each of the eight loses less than 2^-13 of it, so a result's error
# is below the sum over its eights of 8 * 2^-13 of their largest product; beside
# the bar of the 32-bit sums.
@pytest.mark.parametrize("k", [520, 640, 1152, 1500, 2944, 6560])
@pytest.mark.parametrize("m,n", [(5, 70), (300, 700), (690, 700), (990, 1000), (1400, 1390), (1500, 1490)])
def test_parts_of_the_summed_axis(m, n, k):
    """Blocks of 128 that the waves' parts do not divide, parts that begin inside a word of scales."""
    test_product(m, n, k)


@pytest.mark.parametrize("m,n,k", SIZES + [(3000, 4200, 300), (4096, 3600, 1152)])
def test_short_sums(m, n, k):
    torch, D = lib()
    rng = np.random.RandomState(m + n + k)
    a, sa, av = codes(torch, D, operand(rng, m, k))
    b, sb, bv = codes(torch, D, operand(rng, n, k))
    bias, biasv = rounded(torch, rng.randn(n), "f32")
    say(f"[short sums] {m} x {n} x {k}")
    rows, cols = rng.permutation(m)[:150], rng.permutation(n)[:150]     # sampled where there are many
    rows[0], cols[0] = m - 1, n - 1
    ra, rb = av[rows], bv[cols]
    ref = S.product(ra, rb, biasv[cols])
    size = np.sqrt((ra ** 2).sum(axis=1)[:, None] * (rb ** 2).sum(axis=1)[None, :])
    lost = np.zeros_like(ref)
    for i in range(0, ra.shape[1], 8):
        lost += 2.0 ** -10 * (np.abs(ra[:, None, i:i + 8]) * np.abs(rb[None, :, i:i + 8])).max(axis=2)
    for t in ("bf16", "f32"):
        c = torch.full((m, n), float("nan"), device="cuda").to(dtype(torch, t))
        D.dtst_product(a, sa, b, sb, c, bias=bias, short_sums=True)
        got = f64(c)[np.ix_(rows, cols)]
        assert not np.isnan(f64(c)).any()
        tol = HALF_STEP[t] * np.abs(ref) * (1 + 1e-5) + 1e-5 * (np.abs(ref) + size) + lost
        worst = (np.abs(got - ref) / tol).max()
        say(f"  {t}: up to {worst:.2f} of the bar")
        assert worst <= 1


# Large enough for the 8-bit instruction (2^38 operations): each tile, and rows
# and columns that end inside one.
@pytest.mark.parametrize("m,n,k", [(4096, 4100, 8200), (6003, 5000, 5000), (2500, 7777, 8192)])
def test_short_sums_of_large_products(m, n, k):
    torch, D = lib()
    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    x, w = (torch.randn((r, k), generator=g, device="cuda") * torch.exp2(2 * torch.randn((r, 1), generator=g, device="cuda"))
            for r in (m, n))
    a, b = D.empty_codes(m, k), D.empty_codes(n, k)
    D.dtst_quantise(x, *a)
    D.dtst_quantise(w, *b)
    c, e = (torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    D.dtst_product(*a, *b, c, short_sums=True)
    D.dtst_product(*a, *b, e)
    assert not torch.isnan(c).any() and not torch.isnan(e).any()
    rng = np.random.RandomState(k)
    rows, cols = rng.permutation(m)[:120], rng.permutation(n)[:120]
    rows[:2], cols[:2] = (m - 1, 0), (n - 1, 0)

    def values(q, i):
        return S.values(q[0][i].float().cpu().numpy(), q[1].view(torch.uint8)[i].cpu().numpy()[:, :(k + 127) // 128].astype(int) - 127)

    ra, rb = values(a, rows), values(b, cols)
    ref = S.product(ra, rb)
    size = np.sqrt((ra ** 2).sum(axis=1)[:, None] * (rb ** 2).sum(axis=1)[None, :])
    lost = np.zeros_like(ref)
    for i in range(0, ra.shape[1], 8):
        lost += 2.0 ** -10 * (np.abs(ra[:, None, i:i + 8]) * np.abs(rb[None, :, i:i + 8])).max(axis=2)
    for got, name, more in ((f64(c)[np.ix_(rows, cols)], "short", lost), (f64(e)[np.ix_(rows, cols)], "exact", 0.0)):
        tol = HALF_STEP["bf16"] * np.abs(ref) * (1 + 1e-5) + 1e-5 * (np.abs(ref) + size) + more
        worst = (np.abs(got - ref) / tol).max()
        say(f"  {name}: up to {worst:.2f} of the bar")
        assert worst <= 1, name


@pytest.mark.parametrize("m,n,k", [(4097, 6200, 100), (4097, 6200, 700), (8200, 8200, 300), (5000, 5003, 130),
                                   (12000, 4100, 513), (4600, 9000, 1100)])
@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_several_rounds_of_tiles(m, n, k, t):
    """All of the result against a 32-bit product of the values: 2^-22 k / 2 of
    its terms' size each side, and half a unit of the result's type."""
    torch, D = lib()
    g = torch.Generator(device="cuda")
    g.manual_seed(m + k)
    x, w = (torch.randn((r, k), generator=g, device="cuda") * torch.exp2(torch.randn((r, 1), generator=g, device="cuda"))
            for r in (m, n))
    bias = torch.randn(n, generator=g, device="cuda")
    a, b = D.empty_codes(m, k), D.empty_codes(n, k)
    D.dtst_quantise(x, *a)
    D.dtst_quantise(w, *b)

    def values(q, s):
        e = torch.exp2(s.view(torch.uint8)[:, :q.shape[1] // 128].float() - 127)
        return q.float() * e.repeat_interleave(128, dim=1)

    av, bv = values(*a), values(*b)
    c = torch.full((m, n), float("nan"), device="cuda").to(dtype(torch, t))
    D.dtst_product(*a, *b, c, bias=bias)
    ref = av @ bv.t().contiguous() + bias
    size = av.norm(dim=1)[:, None] * bv.norm(dim=1)[None, :] + bias.abs()
    bar = size * (2.0 ** -22 * max(1.0, k / 16)) + (ref.abs() * 2.0 ** -8 if t == "bf16" else 0)
    assert bool(((c.float() - ref).abs() <= bar).all())
    again = torch.full_like(c, float("nan"))
    D.dtst_product(*a, *b, again, bias=bias)
    assert torch.equal(c, again)


@pytest.mark.parametrize("m,n,k", [(5, 70, 300), (70, 90, 700), (300, 520, 256)])
def test_strides(m, n, k):
    torch, D = lib()
    rng = np.random.RandomState(m)
    a, sa, av = codes(torch, D, operand(rng, m, k))
    b, sb, bv = codes(torch, D, operand(rng, n, k))

    def wide(q, extra, fill):
        w = torch.full((q.shape[0], q.shape[1] + extra), fill, dtype=torch.uint8, device="cuda")
        w[:, :q.shape[1]] = q.view(torch.uint8)
        return w.view(q.dtype)[:, :q.shape[1]]

    # codes and scales of no number beside the rows
    a, b, sa, sb = wide(a, 48, 127), wide(b, 16, 127), wide(sa, 4, 255), wide(sb, 8, 255)
    for t in ("bf16", "f32"):
        for offset in (0, 1, 3):
            c, w = strided(torch, torch.zeros((m, n), dtype=dtype(torch, t), device="cuda"), 5, offset)
            D.dtst_product(a, sa, b, sb, c)
            near(f64(c), S.product(av, bv), t, f"{t} offset {offset}")
            assert outside(w, n, offset)


def test_blocks_of_unlike_scales():
    torch, D = lib()
    m, n, k = 20, 140, 1024
    rng = np.random.RandomState(4)
    v = rng.randn(m, k) * np.repeat(np.exp2(rng.randint(-20, 20, (m, 8)).astype(float)), 128, axis=1)
    a, sa, av = codes(torch, D, v)
    b, sb, bv = codes(torch, D, rng.randn(n, k) / np.repeat(np.exp2(rng.randint(-9, 9, (n, 8)).astype(float)), 128, axis=1))
    c = torch.empty((m, n), device="cuda")
    D.dtst_product(a, sa, b, sb, c)
    size = np.abs(av) @ np.abs(bv).T
    near(f64(c) / size, S.product(av, bv) / size, "f32", "unlike scales", rms=1.0)


def test_no_numbers_stay_in_their_rows():
    torch, D = lib()
    x = torch.randn(70, 256, device="cuda")
    x[5, 3] = float("nan")
    w = torch.randn(40, 256, device="cuda")
    w[7, 200] = float("inf")
    a, b = D.empty_codes(70, 256), D.empty_codes(40, 256)
    D.dtst_quantise(x, *a)
    D.dtst_quantise(w, *b)
    c = torch.zeros((70, 40), device="cuda")
    D.dtst_product(*a, *b, c)
    bad = torch.isnan(c)
    assert bad[5].all() and bad[:, 7].all() and int(bad.sum()) == 40 + 70 - 1
    z = torch.empty((70, 0), device="cuda")
    D.dtst_product(*a, b[0][:0], b[1][:0], z)


@pytest.mark.parametrize("m,n,k", [(1, 64, 128), (130, 200, 300), (300, 129, 640)])
def test_a_linear_layers_gradients(m, n, k):
    torch, D = lib()
    rng = np.random.RandomState(n)
    x, xv = rounded(torch, rng.randn(m, k), "bf16")
    w, wv = rounded(torch, rng.randn(n, k) / np.sqrt(k), "f32")
    g, gv = rounded(torch, rng.randn(m, n), "bf16")
    xq, xt, wq, wt, gq, gt = (D.empty_codes(*s) for s in ((m, k), (k, m), (n, k), (k, n), (m, n), (n, m)))
    for t, a, b in ((x, xq, xt), (w, wq, wt), (g, gq, gt)):
        D.dtst_quantise(t, *a, qt=b[0], scale_t=b[1])
    y, g_x, g_w = torch.empty((m, n), device="cuda"), torch.empty((m, k), device="cuda"), torch.empty((n, k), device="cuda")
    D.dtst_product(*xq, *wq, y)
    D.dtst_product(*gq, *wt, g_x)
    D.dtst_product(*gt, *xt, g_w)

    def val(a):
        return S.values(*S.quantise(a))

    near(f64(y), S.product(val(xv), val(wv)), "f32", "y")
    near(f64(g_x), S.product(val(gv), val(wv.T)), "f32", "g_x")
    near(f64(g_w), S.product(val(gv.T), val(xv.T)), "f32", "g_w")
    # and near the gradients of the unquantised layer: e4m3 keeps 4 significant bits, so a
    # value is within 2^-4 of itself and a sum of products within 2 * 2^-4 of their size
    for got, a, b in ((g_x, gv, wv.T), (g_w, gv.T, xv.T)):
        size = np.sqrt((a ** 2).sum(axis=1)[:, None] * (b ** 2).sum(axis=1)[None, :])
        assert (np.abs(f64(got) - a @ b.T) <= (2 ** -3 + 2 ** -8) * size + 1e-6).all()


def test_rows_past_32_bits():
    torch, D = lib()
    m, n, k, ld = 700, 33, 256, 1 << 23
    rng = np.random.RandomState(6)
    a, sa, av = codes(torch, D, operand(rng, m, k))
    b, sb, bv = codes(torch, D, operand(rng, n, k))
    big = torch.empty((m, ld), dtype=torch.uint8, device="cuda")
    big[:, 16:16 + k] = a.view(torch.uint8)
    a2 = big.view(torch.float8_e4m3fn)[:, 16:16 + k]
    for x, sx, xv, y, sy, yv in ((a2, sa, av, b, sb, bv), (b, sb, bv, a2, sa, av)):
        c = torch.empty((x.shape[0], y.shape[0]), device="cuda")
        D.dtst_product(x, sx, y, sy, c)
        near(f64(c), S.product(xv, yv), "f32", "far rows")


def test_the_same_every_time():
    torch, D = lib()
    rng = np.random.RandomState(9)
    for m, n, k in ((3, 500, 4096), (200, 300, 2048), (600, 600, 512)):
        a, sa, _ = codes(torch, D, operand(rng, m, k))
        b, sb, _ = codes(torch, D, operand(rng, n, k))
        c1, c2 = torch.empty((m, n), device="cuda"), torch.empty((m, n), device="cuda")
        D.dtst_product(a, sa, b, sb, c1)
        D.dtst_product(a, sa, b, sb, c2)
        assert torch.equal(c1, c2)
