"""A product's sums are exact to 32 bits, whatever its size and whatever the
caller would put up with."""

import pytest

from gpu_common import say, torch_gpu
from seq_common import dtype

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,n,k", [(5, 70, 1000), (777, 1000, 1900), (4096, 4100, 8200), (6003, 5000, 5000)])
def test_sums_that_may_be_short_are_exact(m, n, k, t):
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    g = torch.Generator(device="cuda")
    g.manual_seed(k)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    a, b = D.empty_codes(m, k), D.empty_codes(n, k)
    D.dtst_quantise(r(m, k), *a)
    D.dtst_quantise(r(n, k), *b)
    bias, base = r(n), r(m, n).to(dtype(torch, t))
    say(f"[product] {m} x {n} x {k} {t}")
    for kw in (dict(), dict(bias=bias), dict(accumulate=True)):
        c, e = base.clone(), base.clone()
        D.dtst_product(*a, *b, c, short_sums=True, **kw)
        D.dtst_product(*a, *b, e, **kw)
        assert torch.equal(c, e), kw
