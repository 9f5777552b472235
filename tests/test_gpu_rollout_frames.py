"""Rollouts of no frames, and of numbers of them that take several plans."""

import numpy as np
import pytest

from gpu_common import torch_gpu
from seq_common import f64, rounded

pytestmark = pytest.mark.gpu

GRID = dict(n_global=(8, 6, 8), n_local=(8, 6, 8), offset=(0, 0, 0), kmax=(1, 1, 2))


def make(torch, B, C=2, F=64):
    from paper_2607_14394_amd.rollout import LatentBlock, Rollout
    rng = np.random.RandomState(1)
    W = 2 * C * 2 * 2 * 4
    w = lambda *s: rounded(torch, rng.randn(*s) / np.sqrt(s[-1]), "f32")[0]  # noqa: E731
    one = torch.ones(W, device="cuda")
    return Rollout(GRID, C, B, [LatentBlock(one, w(3 * F, W), torch.zeros(3 * F, device="cuda"), w(W, F))])


@pytest.mark.parametrize("B,T", [(2, 0), (0, 3), (0, 0)])
def test_no_frames(B, T):
    torch = torch_gpu()
    ro = make(torch, B)
    f = torch.zeros(B, T, 2, 8, 6, 8, device="cuda")
    assert ro.encode(f).shape == (B, T, ro.width)
    before = [s.clone() for s in (ro.reset() or ro.states)]
    assert ro.advance(f).shape == f.shape
    assert all(torch.equal(a, b) for a, b in zip(before, ro.states))
    assert ro.march(f[:, 0] if T else torch.zeros(B, 2, 8, 6, 8, device="cuda"), 0).shape == (B, 0, 2, 8, 6, 8)
    ro.close()


@pytest.mark.parametrize("B,T", [(1, 3), (3, 7), (1, 300), (5, 103)])
def test_frames_by_themselves_and_together(B, T):
    torch = torch_gpu()
    ro = make(torch, B)
    f, _ = rounded(torch, np.random.RandomState(T).randn(B, T, 2, 8, 6, 8), "f32")
    tok = ro.encode(f)
    back = ro.decode(tok)
    for b, t in ((0, 0), (B - 1, T - 1), (B // 2, T // 3)):
        one = ro.encode(f[b:b + 1, t:t + 1])
        assert np.linalg.norm(f64(one[0, 0]) - f64(tok[b, t])) <= 1e-5 * np.linalg.norm(f64(tok[b, t]))
        same = ro.decode(tok[b:b + 1, t:t + 1])
        assert np.linalg.norm(f64(same[0, 0]) - f64(back[b, t])) <= 1e-5 * np.linalg.norm(f64(back[b, t]))
    ro.close()
