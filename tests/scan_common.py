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
