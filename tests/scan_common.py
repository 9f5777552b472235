"""Inputs of the state-space scan's tests (not a test module)."""

import numpy as np

from seq_common import dtype, rounded


def inputs(torch, B, T, F, N, t, seed, lengths=None, gated=True, skip=True, h0=True):
    """Device tensors and their values in 64 bits.  delta, b and c are column
    ranges of one array, the gate of another; what lies past a length is no number."""
    rng = np.random.RandomState(seed)

    def past(v):
        if lengths is not None:
            for i, n in enumerate(lengths):
                v[i, max(0, n):] = np.nan
        return v

    p, pv = rounded(torch, past(np.concatenate([rng.randn(B, T, F) - 2, rng.randn(B, T, 2 * N)], axis=2)), t)
    q, qv = rounded(torch, past(rng.randn(B, T, 2 * F)), t)
    x, xv = rounded(torch, past(rng.randn(B, T, F)), t)
    a, av = rounded(torch, -np.exp(rng.uniform(-2, 2, (N, F))), "f32")
    d, dv = rounded(torch, rng.randn(F), "f32")
    h, hv = rounded(torch, rng.randn(B, N, F), "f32")
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    dev = dict(x=x, delta=p[..., :F], a=a, b=p[..., F:F + N], c=p[..., F + N:], d=d if skip else None,
               o=q[..., F:] if gated else None, h0=h if h0 else None, lengths=n)
    val = dict(x=xv, delta=pv[..., :F], a=av, b=pv[..., F:F + N], c=pv[..., F + N:], d=dv if skip else None,
               o=qv[..., F:] if gated else None, h0=hv if h0 else None, lengths=lengths)
    return dev, val


def empty(torch, like, *shape):
    """As no number, so that what a call leaves out shows."""
    return torch.full(shape, float("nan"), dtype=torch.float32, device="cuda").to(dtype(torch, like))


def divided(D, B, T, F, N):
    """Segments of a sequence forward and backward, and its spans, from the sizes of
    the workspaces: (N + 2, F) of 32 bits a segment forward, and (N + 1, F) more
    backward beside b and c and a tile's sums of 16 steps a span each."""
    spans, tiles = -(-T // D.SCAN_SPAN), -(-F // 64)
    forward = D.dtst_scan_workspace(B, T, F, N) // (B * (N + 2) * F * 4)
    rest = D.dtst_scan_adj_workspace(B, T, F, N) - (tiles + 1) * B * spans * D.SCAN_SPAN * N * 2 * 4
    return max(1, forward), max(1, rest // (B * (2 * N + 3) * F * 4)), spans


# Divided sequences whose segments are of several spans, the last a shorter one: B, T,
# F, N, type, lengths inside, at and past segments' limits (of 64 steps forward and 48
# backward in the first), segments forward and backward.  Workgroups of four waves,
# whose chunks are of 32 steps, in the first, second and fourth, of one and of eight
# steps in the third; 65536 states and more in the first two, whose segments one wave composes,
# and fewer, by eight, in the others.
SPANS = [
    (8, 300, 4096, 12, "f32", None, 5, 7),
    (8, 300, 4096, 16, "bf16", [300, 0, 64, 65, 96, 299, 33, 192], 5, 7),
    (8, 2500, 330, 20, "f16", [2500, 0, 1237, 31, 48, 49, 2496, 5], 53, 79),
    (1, 6000, 1280, 2, "f32", None, 188, 188),
]
