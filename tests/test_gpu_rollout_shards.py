"""Rollouts on shards of a domain: the sum of their coefficients over the shards
makes each one's prediction that of the whole domain."""

import numpy as np
import pytest

from gpu_common import say, torch_gpu
from seq_common import f64, rounded

pytestmark = pytest.mark.gpu


def rel(a, b):
    return float(np.linalg.norm(a - b) / np.linalg.norm(b))


@pytest.mark.parametrize("axis", [0, 1, 2])
def test_two_shards(axis):
    torch = torch_gpu()
    from paper_2607_14394_amd.rollout import LatentBlock, Rollout
    N, K, B, T, C = (16, 12, 20), (2, 3, 2), 2, 4, 2
    W, F = 2 * C * 8 * K[0] * K[1] * K[2], 96
    rng = np.random.RandomState(axis)
    w = lambda *s: rounded(torch, rng.randn(*s) / np.sqrt(s[-1]), "f32")[0]  # noqa: E731
    block = LatentBlock(torch.ones(W, device="cuda"), w(3 * F, W), torch.zeros(3 * F, device="cuda"), w(W, F))
    f, _ = rounded(torch, rng.randn(B, T, C, *N), "f32")
    whole = Rollout(dict(n_global=N, n_local=N, offset=(0, 0, 0), kmax=K), C, B, [block])
    tokens, ahead = whole.encode(f), whole.advance(f)
    cut = N[axis] // 2 + 1
    parts = []
    shards = [(slice(0, cut), cut, 0), (slice(cut, None), N[axis] - cut, cut)]
    ros = []
    for here, n, at in shards:
        grid = dict(n_global=N, n_local=tuple(n if i == axis else N[i] for i in range(3)),
                    offset=tuple(at if i == axis else 0 for i in range(3)), kmax=K)
        ros.append(Rollout(grid, C, B, [block], reduce=lambda t: parts.append(t.clone())))
        ros[-1].encode(f[(slice(None),) * (3 + axis) + (here,)])
    total = parts[0] + parts[1]
    # the two sums over the shards differ from the whole's by their order
    assert rel(f64(total), f64(tokens)) <= 1e-5
    assert rel(f64(parts[0]), f64(tokens)) > 0.1     # (what one shard has is another thing)
    for (here, _, _), ro in zip(shards, ros):
        ro.reduce = lambda t: t.copy_(total)
        got = ro.advance(f[(slice(None),) * (3 + axis) + (here,)])
        want = ahead[(slice(None),) * (3 + axis) + (here,)]
        say(f"[shards] axis {axis}: rel {rel(f64(got), f64(want)):.2e}")
        assert got.shape == want.shape and rel(f64(got), f64(want)) <= 2.0 ** -7   # (one bf16 step, as between the block's forms)
        ro.close()
    whole.close()
