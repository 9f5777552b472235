"""What the binding of the operators on latent sequences refuses: other types,
shapes, devices, and tensors whose rows are not contiguous, single rows too."""

import pytest

from gpu_common import torch_gpu

pytestmark = pytest.mark.gpu


def lib():
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    return torch, D


def new(torch, *shape, dtype=None):
    return torch.zeros(shape, dtype=dtype or torch.bfloat16, device="cuda")


def every_other(torch, t):
    """t's shape and type, every other element of longer rows."""
    wide = torch.zeros(t.shape[:-1] + (2 * t.shape[-1],), dtype=torch.uint8, device="cuda").to(torch.float32)
    return wide.to(t.dtype)[..., ::2]


@pytest.mark.parametrize("rows", [1, 3])
def test_norm(rows):
    torch, D = lib()
    f32 = torch.float32
    x, w, y = new(torch, rows, 256), new(torch, 256, dtype=f32), new(torch, rows, 256)
    q, s = D.empty_codes(rows, 256)
    D.dtst_rms_norm(x, w, y)
    D.dtst_rms_norm(x, w, q, scale=s)
    for bad in (dict(x=every_other(torch, x)), dict(y=every_other(torch, y)), dict(w=every_other(torch, w)),
                dict(x=x.double()), dict(y=y.float()), dict(w=w.half()), dict(x=x.cpu()), dict(x=x[None]),
                dict(y=new(torch, rows + 1, 256)), dict(res=new(torch, rows, 255)), dict(res=x.half()),
                dict(sum_out=every_other(torch, x)), dict(rstd=new(torch, rows + 1, dtype=f32)),
                dict(y=q, scale=s[:, :1]), dict(y=q[:, :128], scale=s),
                dict(y=q, scale=torch.zeros(rows, 8, dtype=torch.uint8, device="cuda").view(s.dtype)[:, ::2]),
                dict(y=torch.zeros(rows, 512, dtype=torch.uint8, device="cuda").view(q.dtype)[:, ::2], scale=s)):
        a = dict(dict(x=x, w=w, y=y), **bad)
        with pytest.raises(ValueError):
            D.dtst_rms_norm(a.pop("x"), a.pop("w"), a.pop("y"), **a)


@pytest.mark.parametrize("m", [1, 3])
def test_product(m):
    torch, D = lib()
    a, b, c = D.empty_codes(m, 200), D.empty_codes(64, 200), new(torch, m, 64)
    for t in (*a, *b):
        t.view(torch.uint8).fill_(120)
    D.dtst_product(*a, *b, c)
    u8 = torch.uint8
    gaps = torch.zeros(m, 512, dtype=u8, device="cuda").view(a[0].dtype)[:, ::2]
    gaps_s = torch.zeros(m, 8, dtype=u8, device="cuda").view(a[1].dtype)[:, ::2]
    for args in ((gaps, a[1], *b, c), (a[0], gaps_s, *b, c), (a[0].view(u8), a[1], *b, c), (a[0], a[1].view(u8), *b, c),
                 (*a, *b, every_other(torch, c)), (*a, *b, c.double()), (*a, *b, new(torch, m + 1, 64)),
                 (a[0][:, :100], a[1], *b, c), (*a, b[0].cpu(), b[1], c)):
        with pytest.raises(ValueError):
            D.dtst_product(*args)
    with pytest.raises(ValueError):
        D.dtst_product(*a, *b, c, bias=new(torch, 63, dtype=torch.float32))
    x = new(torch, m, 200)
    for kw in (dict(q=a[0]), dict(scale=a[1]), dict(), dict(q=gaps, scale=a[1]), dict(q=a[0], scale=gaps_s),
               dict(q=b[0], scale=b[1])):
        with pytest.raises(ValueError):
            D.dtst_quantise(x, **kw)
    with pytest.raises(ValueError):
        D.dtst_quantise(every_other(torch, x), *a)


def test_recurrence():
    torch, D = lib()
    f32 = torch.float32
    z, v, y, h = new(torch, 2, 5, 8), new(torch, 2, 5, 8), new(torch, 2, 5, 8), new(torch, 2, 8, dtype=f32)
    D.dtst_recurrence(z, v, y, h0=h, h_out=h)
    for bad in (dict(z=z.float()), dict(z=z[0]), dict(v=every_other(torch, v)), dict(y=new(torch, 2, 6, 8)), dict(v=v.cpu()),
                dict(o=new(torch, 2, 5, 7)), dict(h0=new(torch, 2, 7, dtype=f32)), dict(h0=h.half()),
                dict(h_out=every_other(torch, h)), dict(states=new(torch, 2, 2, 8, dtype=f32)),
                dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")),
                dict(lengths=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        a = dict(dict(z=z, v=v, y=y), **bad)
        with pytest.raises(ValueError):
            D.dtst_recurrence(a.pop("z"), a.pop("v"), a.pop("y"), **a)
    st = new(torch, *D.recurrence_states_shape(2, 5, 8), dtype=f32)
    with pytest.raises(ValueError):
        D.dtst_recurrence_adj(z, v, y, st, new(torch, 2, 5, 8), new(torch, 2, 5, 8), o=v)
    with pytest.raises(ValueError):
        D.dtst_recurrence_adj(z, v, y, st[:, :, :7], new(torch, 2, 5, 8), new(torch, 2, 5, 8))


def test_workspaces():
    """One on the host, with gaps, too small or at an odd address is refused."""
    torch, D = lib()
    f32, u8 = torch.float32, torch.uint8
    z, v, y = new(torch, 1, 300, 8), new(torch, 1, 300, 8), new(torch, 1, 300, 8)
    need = D.dtst_recurrence_workspace(1, 300, 8, z.dtype)
    good = torch.empty(need, dtype=u8, device="cuda")
    D.dtst_recurrence(z, v, y, ws=good)
    g, w, g_w = new(torch, 5, 64), new(torch, 64, dtype=f32), new(torch, 64, dtype=f32)
    rstd = new(torch, 5, dtype=f32)
    need_n = D.dtst_rms_norm_adj_workspace(5, 64)
    D.dtst_rms_norm_adj(g, new(torch, 5, 64), w, rstd, new(torch, 5, 64), g_w, ws=torch.empty(need_n, dtype=u8, device="cuda"))
    for n, call in ((need, lambda ws: D.dtst_recurrence(z, v, y, ws=ws)),
                    (need_n, lambda ws: D.dtst_rms_norm_adj(g, new(torch, 5, 64), w, rstd, new(torch, 5, 64), g_w, ws=ws))):
        wide = torch.empty(2 * n + 16, dtype=u8, device="cuda")
        for bad in (torch.empty(n, dtype=u8), wide[:2 * n:2]):
            with pytest.raises(ValueError):
                call(bad)
        for bad in (wide[:n - 1], wide[1:n + 1]):
            with pytest.raises(D.DtstError):
                call(bad)
