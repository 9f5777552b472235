"""Views of one array as operands: those that share an element are refused, all
others are taken."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def whole(torch, D, z, v):
    """The same from arrays of their own."""
    y = torch.empty(z.shape, dtype=z.dtype, device="cuda")
    D.dtst_recurrence(z.contiguous(), v.contiguous(), y)
    return y


def test_steps_and_entries_of_one_array():
    torch, D = lib()
    B, T, F = 3, 40, 72
    a = torch.randn(B, 3 * T, F, device="cuda")
    b = torch.randn(B, T, 3, F, device="cuda")
    c = torch.randn(3 * B, T, F, device="cuda")
    d = torch.randn(T, B, 3 * F, device="cuda").transpose(0, 1)
    for name, z, v, y in (("runs of steps", a[:, :T], a[:, T:2 * T], a[:, 2 * T:]),
                          ("every third step", b[:, :, 0], b[:, :, 1], b[:, :, 2]),
                          ("runs of entries", c[:B], c[B:2 * B], c[2 * B:]),
                          ("every third entry", c[::3], c[1::3], c[2::3]),
                          ("columns, steps first", d[..., :F], d[..., F:2 * F], d[..., 2 * F:])):
        say(f"[views] {name}")
        want = whole(torch, D, z, v)
        D.dtst_recurrence(z, v, y)
        assert torch.equal(y, want), name
    for z, v, y in ((a[:, :T], a[:, T:2 * T], a[:, 2 * T - 1:3 * T - 1]), (c[:B], c[B:2 * B], c[B - 1:2 * B - 1]),
                    (d[..., :F], d[..., F:2 * F], d[..., 2 * F - 1:3 * F - 1])):
        with pytest.raises(D.DtstError, match="overlap"):
            D.dtst_recurrence(z, v, y)


def test_random_views():
    torch, D = lib()
    rng = np.random.RandomState(3)
    a = torch.randn(4000, device="cuda")
    ids = np.arange(4000)
    v0 = torch.randn(5 * 6 * 9, device="cuda")
    taken = refused = 0
    for _ in range(500):
        B, T, F = rng.randint(1, 5), rng.randint(1, 6), rng.randint(1, 9)
        if rng.rand() < 0.5:
            st = F + rng.randint(0, 3)
            sb = T * st + rng.randint(0, 20)
        else:
            sb = F + rng.randint(0, 3)
            st = B * sb + rng.randint(0, 20)
        at = 500 + rng.randint(-200, 200)
        views = [torch.as_strided(a, (B, T, F), (sb, st, 1), o) for o in (500, at)]
        where = [set(np.lib.stride_tricks.as_strided(ids[o:], (B, T, F), (sb * 8, st * 8, 8)).ravel()) for o in (500, at)]
        z, y = views
        v = v0[:B * T * F].view(B, T, F)
        if where[0] & where[1]:
            refused += 1
            before = a.clone()
            with pytest.raises(D.DtstError, match="overlap"):
                D.dtst_recurrence(z, v, y)
            assert torch.equal(a, before)
        else:
            taken += 1
            want = whole(torch, D, z, v)
            D.dtst_recurrence(z, v, y)
            assert torch.equal(y, want)
    say(f"[views] {taken} taken, {refused} refused")
    assert taken > 50 and refused > 50


def test_states_between_the_rows():
    """A state that lies in the columns which the steps leave free is taken, in
    place too; one that reaches into them is refused."""
    torch, D = lib()
    T, F = 300, 64
    a = torch.randn(1, T, 4 * F, device="cuda")
    z, v, y, free = (a[..., i * F:(i + 1) * F] for i in range(4))
    want, last = torch.empty(1, T, F, device="cuda"), torch.empty(1, F, device="cuda")
    h0 = free[:, 7].clone()
    D.dtst_recurrence(z.contiguous(), v.contiguous(), want, h0=h0, h_out=last)
    h = free[:, 7]
    D.dtst_recurrence(z, v, y, h0=h, h_out=h)
    assert torch.equal(y, want) and torch.equal(h, last)
    with pytest.raises(D.DtstError, match="y and h_out"):
        D.dtst_recurrence(z, v, y, h_out=a[:, 7, 3 * F - 1:4 * F - 1])


def test_vectors_between_the_rows():
    """The norm's weight, 1 / rms and single rows in the columns that other
    operands leave free."""
    torch, D = lib()
    R, C = 9, 64
    a = torch.randn(R, 4 * C, device="cuda")
    x, y, u, free = (a[:, i * C:(i + 1) * C] for i in range(4))
    w, rstd, want, r1 = free[2], free[3, :R], torch.empty(R, C, device="cuda"), torch.empty(R, device="cuda")
    D.dtst_rms_norm(x.contiguous(), w.clone(), want, rstd=r1)
    D.dtst_rms_norm(x, w, y, sum_out=u, rstd=rstd)
    assert torch.equal(y, want) and torch.equal(rstd, r1) and torch.equal(u, x)
    g_u, g_w, g_u1, g_w1 = (torch.empty(*s, device="cuda") for s in ((R, C), (C,), (R, C), (C,)))
    ws = torch.empty(D.dtst_rms_norm_adj_workspace(R, C), dtype=torch.uint8, device="cuda")
    D.dtst_rms_norm_adj(y, u, w, rstd, g_u, free[4], ws=ws)
    D.dtst_rms_norm_adj(y.contiguous(), u.contiguous(), w.clone(), r1, g_u1, g_w1)
    assert torch.equal(g_u, g_u1) and torch.equal(free[4], g_w1)
    with pytest.raises(D.DtstError, match="y and weight"):
        D.dtst_rms_norm(x, a[2, C + 1:2 * C + 1], y)
    with pytest.raises(D.DtstError, match="rstd and x"):
        D.dtst_rms_norm(x, w, y, rstd=a.view(-1)[2 * 4 * C - 3:2 * 4 * C - 3 + R])
