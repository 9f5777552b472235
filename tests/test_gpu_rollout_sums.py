"""The sums of a block's products do not go by the batch it runs in."""

import pytest

from gpu_common import say, torch_gpu

pytestmark = pytest.mark.gpu


def test_a_large_block_takes_the_sums_of_a_small_one():
    """Sequences by themselves and among others (2^39 operations in the first
    product): the same states and branches but for the order of 32-bit sums,
    which another tile may take; 2^-9 of a bf16 result changes then at most
    rarely.  Sums of 13 bits change one result in 250."""
    torch = torch_gpu()
    import paper_2607_14394_amd as D
    from paper_2607_14394_amd.rollout import LatentBlock
    B, T, W, F = 256, 160, 2048, 2048
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    block = LatentBlock(torch.ones(W, device="cuda"), r(3 * F, W) / W ** 0.5, torch.zeros(3 * F, device="cuda"), r(W, F) / F ** 0.5)
    x = r(B, T, W).to(torch.bfloat16)
    out, _ = block.forward(x, None)
    # the same from the library's calls with exact sums
    R, bf = B * T, torch.bfloat16
    n, yq = D.empty_codes(R, W), D.empty_codes(R, F)
    p, y, want = (torch.empty(s, dtype=bf, device="cuda") for s in ((B, T, 3 * F), (B, T, F), (B, T, W)))
    D.dtst_rms_norm(x.view(R, W), block.norm, n[0], sum_out=torch.empty((R, W), device="cuda"), scale=n[1], eps=block.eps)
    D.dtst_product(*n, *block.w_in.rows, p.view(R, 3 * F), bias=block.b_in)
    D.dtst_recurrence(p[..., :F], p[..., F:2 * F], y, o=p[..., 2 * F:])
    D.dtst_quantise(y.view(R, F), *yq)
    D.dtst_product(*yq, *block.w_out.rows, want.view(R, W))
    assert torch.equal(out, want)
    few, _ = block.forward(x[:2].contiguous(), None)
    changed = float((few != out[:2]).float().mean())
    say(f"[block] {changed:.1e} of the results differ in a batch of {B}")
    assert changed <= 2.0 ** -9
