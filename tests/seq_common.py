"""Helpers of the latent-sequence operators' tests (not a test module)."""

import numpy as np

# Half the step between neighbouring values of a type, relative to the value
# (f16 also has a smallest step): what one rounding may add.
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
LEAST = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}


def dtype(torch, t):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def f64(t):
    """A device tensor as a float64 array."""
    return t.detach().float().cpu().double().numpy() if t.dtype.itemsize < 4 else t.detach().cpu().double().numpy()


def rounded(torch, a, t):
    """An array rounded to a type, as a device tensor and as float64."""
    d = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float64)).to(dtype(torch, t)).cuda()
    return d, f64(d)


def near(got, ref, t, name, arithmetic=1e-5, rms=None):
    """Every value within one rounding to its type and `arithmetic` (the fp32
    path's bar, relative to the value and to the RMS) of the oracle's."""
    got, ref = np.asarray(got, np.float64), np.asarray(ref, np.float64)
    assert got.shape == ref.shape, (name, got.shape, ref.shape)
    if ref.size == 0:
        return
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{name}: no numbers in other places"
    ok = ~np.isnan(ref)
    got, ref = got[ok], ref[ok]
    rms = np.sqrt((ref ** 2).mean()) if rms is None else rms
    tol = HALF_STEP[t] * np.abs(ref) * (1 + 1e-5) + LEAST[t] + arithmetic * (np.abs(ref) + rms)
    off = np.abs(got - ref) - tol
    worst = np.abs(got - ref).max() if ref.size else 0.0
    print(f"  {name}: max difference {worst:.2e}, rms {rms:.2e}", flush=True)
    assert (off <= 0).all(), f"{name}: {int((off > 0).sum())} of {off.size} values off, by up to {off.max():.3e}"


def strided(torch, d, extra=0, offset=0):
    """The same values as a view with contiguous last axis and wider rows,
    starting `offset` elements into its memory, surrounded by no-numbers."""
    shape = d.shape[:-1] + (d.shape[-1] + extra + offset,)
    w = torch.full(shape, float("nan"), dtype=torch.float32).to(d.dtype).to(d.device)
    v = w[..., offset:offset + d.shape[-1]]
    v.copy_(d)
    return v, w


def outside(w, width, offset):
    """Whether everything beside a strided output is still no number."""
    import torch
    return bool(torch.isnan(w[..., :offset].float()).all()) and bool(torch.isnan(w[..., offset + width:].float()).all())
