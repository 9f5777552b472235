"""Marching fields in time past a plan's window: every time step's retained
coefficients (one batch entry of a plan with a single time step) are a token,
residual blocks with a recurrence run over the sequence of tokens, and the result
is expanded back onto the shard.  A block is either of

    u = x + residual;  n = rms norm of u;  z | v | o = n W_in^T + b
    y = recurrence(z, v, o);  x' = y W_out^T;  residual' = u

    u = x + residual;  n = layer norm of u;  s | o = n W_in^T + b
    v = convolution(s);  delta | b | c = v W_x^T + b_x
    y = scan(v, delta, a, b, c, d, o);  x' = y W_out^T;  residual' = u

Orchestration only: every step is a call of the DTST library
(``dtst_rms_norm``, ``dtst_layer_norm``, ``dtst_quantise``, ``dtst_product``,
``dtst_recurrence``, ``dtst_conv``, ``dtst_scan``, their backward calls,
``dtst_global_norm``, ``dtst_clip`` and the plan's transforms), apart from the last
residual's addition, the sum of a bias' gradient, and in training with lengths the
clearing of what lies past them.  Weights are kept in 8 bits with their
transposes, as the backward needs them; the masters stay with the caller.
"""

from __future__ import annotations

import torch

from . import (DtstError, Plan, dtst_clip, dtst_conv, dtst_conv_adj, dtst_conv_adj_workspace, dtst_desc_validate,
               dtst_global_norm, dtst_layer_norm, dtst_layer_norm_adj, dtst_layer_norm_adj_workspace, dtst_product,
               dtst_quantise, dtst_recurrence, dtst_recurrence_adj, dtst_rms_norm, dtst_rms_norm_adj,
               dtst_rms_norm_adj_workspace, dtst_scan, dtst_scan_adj, dtst_scan_workspace, empty_codes,
               recurrence_states_shape, scan_states_shape)

_UNSUPPORTED = 2  # DTST_ERR_UNSUPPORTED


def _past(lengths, steps):
    """(B T, 1), true where a step lies past its sequence's length."""
    return (torch.arange(steps, device=lengths.device) >= lengths[:, None]).view(len(lengths) * steps, 1)


class _Weights:
    """A linear layer's weights (out, in) as codes, along both axes."""

    def __init__(self, w):
        out, k = w.shape
        self.shape = (out, k)
        self.rows, self.cols = empty_codes(out, k, w.device), empty_codes(k, out, w.device)
        self.set(w)

    def set(self, w):
        dtst_quantise(w, *self.rows, qt=self.cols[0], scale_t=self.cols[1])


def _both(t):
    """The codes of t's rows and of its transpose's."""
    r, c = t.shape
    q, qt = empty_codes(r, c, t.device), empty_codes(c, r, t.device)
    dtst_quantise(t, *q, qt=qt[0], scale_t=qt[1])
    return q, qt


def _weight_gradient(qt, xt, rows, g):
    """The sum over `rows` tokens; a product has to have something to sum."""
    if rows:
        dtst_product(*qt, *xt, g)
    else:
        g.zero_()


class LatentBlock:
    """One residual block of width W (32768 at most, the norm's limit) with F
    recurrent features.  norm: (W,) float32; w_in: (3 F, W); b_in: (3 F,)
    float32; w_out: (W, F)."""

    def __init__(self, norm, w_in, b_in, w_out, eps=1e-6):
        self.width, self.features = w_out.shape
        if tuple(w_in.shape) != (3 * self.features, self.width) or tuple(norm.shape) != (self.width,):
            raise ValueError(f"w_out {tuple(w_out.shape)} needs w_in ({3 * self.features}, {self.width}) and norm "
                             f"({self.width},)")
        try:
            dtst_rms_norm_adj_workspace(1, self.width)
        except DtstError as e:  # (here, rather than at the first forward)
            raise ValueError(f"a block of width {self.width}: {e}") from None
        self.norm, self.b_in, self.eps = norm, b_in, eps
        self.w_in, self.w_out = _Weights(w_in), _Weights(w_out)

    def set_weights(self, w_in, w_out):
        """New weights of the same shapes (after an update of the masters)."""
        self.w_in.set(w_in)
        self.w_out.set(w_out)

    def state(self, batch, device="cuda"):
        """The state before the first step."""
        return torch.zeros((batch, self.features), dtype=torch.float32, device=device)

    def _split(self, p):
        F = self.features
        return p[..., :F], p[..., F:2 * F], p[..., 2 * F:]

    def forward(self, x, res, state=None, lengths=None, keep=None):
        """x: (B, T, W), the branch of the block before (bfloat16, or float32
        for the first); res: (B, T, W) float32 or None, updated in place unless
        `keep` is given.  Returns the block's branch (bfloat16) and the residual.
        state: (B, F) float32, updated in place; one step with a state is a
        serving step.  keep: a dict that receives what backward needs.
        Past a sequence's length (B,) int32 x and res may hold anything."""
        B, T, W = x.shape
        F, R, dev = self.features, B * T, x.device
        bf = torch.bfloat16
        x2 = x.reshape(R, W)
        u = torch.empty((R, W), dtype=torch.float32, device=dev) if res is None else res.view(R, W)
        res2 = None if res is None else u
        n = empty_codes(R, W, dev)
        p, y = torch.empty((B, T, 3 * F), dtype=bf, device=dev), torch.empty((B, T, F), dtype=bf, device=dev)
        z, v, o = self._split(p)
        states = None
        if keep is None:
            dtst_rms_norm(x2, self.norm, n[0], res=res2, sum_out=u, scale=n[1], eps=self.eps)
        else:
            rstd, nt = torch.empty(R, dtype=torch.float32, device=dev), empty_codes(W, R, dev)
            plain = torch.empty((R, W), dtype=x.dtype, device=dev)
            u = u if res is None else torch.empty_like(u)  # (the caller's stays: backward needs this one)
            dtst_rms_norm(x2, self.norm, plain, res=res2, sum_out=u, rstd=rstd, eps=self.eps)
            kept_u, past = u, None if lengths is None else _past(lengths, T)
            if past is not None:
                # The weights' gradients sum over the rows, and the transposed
                # form scales 128 of them at once: what lies past a length would
                # reach the others there, and zero times no number is none.
                plain.masked_fill_(past, 0)
                rstd.masked_fill_(past[:, 0], 0)
                kept_u = u.masked_fill(past, 0)
            dtst_quantise(plain, *n, qt=nt[0], scale_t=nt[1])
            states = torch.empty(recurrence_states_shape(B, T, F), dtype=torch.float32, device=dev)
            keep.update(shape=(B, T), u=kept_u, rstd=rstd, nt=nt, p=p, states=states, lengths=lengths, past=past,
                        x_dtype=x.dtype)
        dtst_product(*n, *self.w_in.rows, p.view(R, 3 * F), bias=self.b_in)
        dtst_recurrence(z, v, y, o=o, h0=state, h_out=state, lengths=lengths, states=states)
        yq = empty_codes(R, F, dev)
        if keep is None:
            dtst_quantise(y.view(R, F), *yq)
        else:
            keep["yt"] = empty_codes(F, R, dev)
            dtst_quantise(y.view(R, F), *yq, qt=keep["yt"][0], scale_t=keep["yt"][1])
        out = torch.empty((B, T, W), dtype=bf, device=dev)
        dtst_product(*yq, *self.w_out.rows, out.view(R, W))
        return out, u.view(B, T, W)

    def backward(self, kept, g_out, g_res, g_state=None):
        """Gradients from those of the branch (B, T, W) bfloat16, of the
        residual (B, T, W) float32 and of the last state (B, F), or None.
        Returns a dict: x (in x's type), res (float32), state, norm, w_in, b_in,
        w_out (float32)."""
        B, T = kept["shape"]
        W, F, R, dev = self.width, self.features, B * T, g_out.device
        f32, bf = torch.float32, torch.bfloat16
        go = g_out.reshape(R, W)
        if kept["past"] is not None:
            go = go.masked_fill(kept["past"], 0)  # (as in forward)
        q, qt = _both(go)
        g_y, g_w_out = torch.empty((B, T, F), dtype=bf, device=dev), torch.empty((W, F), dtype=f32, device=dev)
        dtst_product(*q, *self.w_out.cols, g_y.view(R, F))
        _weight_gradient(qt, kept["yt"], R, g_w_out)
        g_p = torch.empty((B, T, 3 * F), dtype=bf, device=dev)
        g_h = torch.empty((B, F), dtype=f32, device=dev)
        z, v, o = self._split(kept["p"])
        g_z, g_v, g_o = self._split(g_p)
        dtst_recurrence_adj(z, v, g_y, kept["states"], g_z, g_v, o=o, g_o=g_o, g_h=g_state, g_hzero=g_h,
                            lengths=kept["lengths"])
        q, qt = _both(g_p.view(R, 3 * F))
        g_n = torch.empty((R, W), dtype=kept["x_dtype"], device=dev)
        g_w_in = torch.empty((3 * F, W), dtype=f32, device=dev)
        dtst_product(*q, *self.w_in.cols, g_n)
        _weight_gradient(qt, kept["nt"], R, g_w_in)
        g_u, g_norm = torch.empty((R, W), dtype=f32, device=dev), torch.empty_like(self.norm)
        g_x = g_u if kept["x_dtype"] == f32 else torch.empty((R, W), dtype=kept["x_dtype"], device=dev)
        dtst_rms_norm_adj(g_n, kept["u"], self.norm, kept["rstd"], g_u, g_norm,
                          g_sum=None if g_res is None else g_res.reshape(R, W), g_x=None if g_x is g_u else g_x)
        return dict(x=g_x.view(B, T, W), res=g_u.view(B, T, W), state=g_h, norm=g_norm, w_in=g_w_in,
                    b_in=g_p.float().sum(dim=(0, 1)), w_out=g_w_out)


class SelectiveBlock:
    """One residual block of width W (32768 at most, the norm's limit) with F
    features of N states (64 at most) behind a convolution of K taps (8 at most).
    norm, norm_bias: (W,) float32; w_in: (2 F, W); b_in: (2 F,); conv: (K, F),
    conv_bias: (F,); w_x: (F + 2 N, F); b_x: (F + 2 N,), its first F the steps' raw
    sizes; a: (N, F), negative; d: (F,); w_out: (W, F).  All but the linear layers'
    weights are float32 and used as given."""

    def __init__(self, norm, norm_bias, w_in, b_in, conv, conv_bias, w_x, b_x, a, d, w_out, eps=1e-5):
        self.width, self.features = w_out.shape
        W, F, N, K = self.width, self.features, a.shape[0], conv.shape[0]
        for t, shape, name in ((norm, (W,), "norm"), (norm_bias, (W,), "norm_bias"), (w_in, (2 * F, W), "w_in"),
                               (b_in, (2 * F,), "b_in"), (conv, (K, F), "conv"), (conv_bias, (F,), "conv_bias"),
                               (w_x, (F + 2 * N, F), "w_x"), (b_x, (F + 2 * N,), "b_x"), (a, (N, F), "a"), (d, (F,), "d")):
            if tuple(t.shape) != shape:
                raise ValueError(f"w_out {(W, F)}, {N} states and {K} taps need {name} {shape}, got {tuple(t.shape)}")
        try:  # (here, rather than at the first forward)
            dtst_layer_norm_adj_workspace(1, W)
            dtst_conv_adj_workspace(1, 1, F, K)
            dtst_scan_workspace(1, 1, F, N)
        except DtstError as e:
            raise ValueError(f"a block of width {W}, {N} states and {K} taps: {e}") from None
        self.states, self.taps, self.eps = N, K, eps
        self.norm, self.norm_bias, self.b_in, self.conv, self.conv_bias = norm, norm_bias, b_in, conv, conv_bias
        self.b_x, self.a, self.d = b_x, a, d
        self.w_in, self.w_x, self.w_out = _Weights(w_in), _Weights(w_x), _Weights(w_out)

    def set_weights(self, w_in, w_x, w_out):
        """New weights of the same shapes (after an update of the masters)."""
        self.w_in.set(w_in)
        self.w_x.set(w_x)
        self.w_out.set(w_out)

    def state(self, batch, device="cuda"):
        """The state before the first step: the convolution's last inputs and the scan's states."""
        return (torch.zeros((batch, self.taps - 1, self.features), dtype=torch.bfloat16, device=device),
                torch.zeros((batch, self.states, self.features), dtype=torch.float32, device=device))

    def _split(self, p):
        F, N = self.features, self.states
        return p[..., :F], p[..., F:F + N], p[..., F + N:]

    def forward(self, x, res, state=None, lengths=None, keep=None):
        """As LatentBlock.forward; state: what `state` gives, updated in place."""
        B, T, W = x.shape
        F, N, R, dev = self.features, self.states, B * T, x.device
        bf = torch.bfloat16
        x2 = x.reshape(R, W)
        u = torch.empty((R, W), dtype=torch.float32, device=dev) if res is None else res.view(R, W)
        res2 = None if res is None else u
        n = empty_codes(R, W, dev)
        s, v, y = (torch.empty((B, T, k * F), dtype=bf, device=dev) for k in (2, 1, 1))
        p = torch.empty((B, T, F + 2 * N), dtype=bf, device=dev)
        inputs, h = (None, None) if state is None else state
        states = None
        if keep is None:
            dtst_layer_norm(x2, self.norm, self.norm_bias, n[0], res=res2, sum_out=u, scale=n[1], eps=self.eps)
        else:
            mean, rstd = (torch.empty(R, dtype=torch.float32, device=dev) for _ in range(2))
            nt, plain = empty_codes(W, R, dev), torch.empty((R, W), dtype=x.dtype, device=dev)
            u = u if res is None else torch.empty_like(u)  # (the caller's stays: backward needs this one)
            dtst_layer_norm(x2, self.norm, self.norm_bias, plain, res=res2, sum_out=u, mean=mean, rstd=rstd, eps=self.eps)
            kept_u, past = u, None if lengths is None else _past(lengths, T)
            if past is not None:  # (as in LatentBlock.forward)
                plain.masked_fill_(past, 0)
                mean.masked_fill_(past[:, 0], 0)
                rstd.masked_fill_(past[:, 0], 0)
                kept_u = u.masked_fill(past, 0)
            dtst_quantise(plain, *n, qt=nt[0], scale_t=nt[1])
            states = torch.empty(scan_states_shape(B, T, F, N), dtype=torch.float32, device=dev)
            keep.update(shape=(B, T), u=kept_u, mean=mean, rstd=rstd, nt=nt, s=s, v=v, p=p, states=states, lengths=lengths,
                        past=past, x_dtype=x.dtype, inputs=None if inputs is None else inputs.clone())
        dtst_product(*n, *self.w_in.rows, s.view(R, 2 * F), bias=self.b_in)
        dtst_conv(s[..., :F], self.conv, v, bias=self.conv_bias, state=inputs, state_out=inputs, lengths=lengths)
        vq = self._codes(v.view(R, F), keep, "vt")
        dtst_product(*vq, *self.w_x.rows, p.view(R, F + 2 * N), bias=self.b_x)
        delta, b, c = self._split(p)
        dtst_scan(v, delta, self.a, b, c, y, d=self.d, o=s[..., F:], h0=h, h_out=h, lengths=lengths, states=states)
        yq = self._codes(y.view(R, F), keep, "yt")
        out = torch.empty((B, T, W), dtype=bf, device=dev)
        dtst_product(*yq, *self.w_out.rows, out.view(R, W))
        return out, u.view(B, T, W)

    @staticmethod
    def _codes(t, keep, name):
        """t's codes, its transpose's kept for the backward."""
        if keep is None:
            q = empty_codes(*t.shape, t.device)
            dtst_quantise(t, *q)
            return q
        q, keep[name] = _both(t)
        return q

    def backward(self, kept, g_out, g_res, g_state=None):
        """As LatentBlock.backward; g_state: the gradients of the state's two parts
        after the last step, or None.  Returns a dict: x (in x's type), res, state (of
        the two parts before the first step), and those of the constructor's arguments
        (float32)."""
        B, T = kept["shape"]
        W, F, N, R, dev = self.width, self.features, self.states, B * T, g_out.device
        f32, bf = torch.float32, torch.bfloat16
        g_inputs_out, g_h_out = (None, None) if g_state is None else g_state
        s, v, lengths = kept["s"], kept["v"], kept["lengths"]
        go = g_out.reshape(R, W)
        if kept["past"] is not None:
            go = go.masked_fill(kept["past"], 0)
        q, qt = _both(go)
        g_y, g_v = (torch.empty((B, T, F), dtype=bf, device=dev) for _ in range(2))
        g_w_in, g_w_x, g_w_out, g_conv, g_a = (torch.empty(k, dtype=f32, device=dev) for k in
                                               ((2 * F, W), (F + 2 * N, F), (W, F), self.conv.shape, (N, F)))
        g_conv_bias, g_d = (torch.empty(F, dtype=f32, device=dev) for _ in range(2))
        dtst_product(*q, *self.w_out.cols, g_y.view(R, F))
        _weight_gradient(qt, kept["yt"], R, g_w_out)
        g_s, g_p = torch.empty_like(s), torch.empty_like(kept["p"])
        g_h = torch.empty((B, N, F), dtype=f32, device=dev)
        g_inputs = torch.empty((B, self.taps - 1, F), dtype=bf, device=dev)
        g_delta, g_b, g_c = self._split(g_p)
        delta, b, c = self._split(kept["p"])
        dtst_scan_adj(v, delta, self.a, b, c, g_y, kept["states"], g_v, g_delta, g_a, g_b, g_c, d=self.d, g_d=g_d,
                      o=s[..., F:], g_o=g_s[..., F:], g_h=g_h_out, g_hzero=g_h, lengths=lengths)
        q, qt = _both(g_p.view(R, F + 2 * N))
        dtst_product(*q, *self.w_x.cols, g_v.view(R, F), accumulate=True)
        _weight_gradient(qt, kept["vt"], R, g_w_x)
        dtst_conv_adj(s[..., :F], self.conv, g_v, g_s[..., :F], g_conv, bias=self.conv_bias, g_bias=g_conv_bias,
                      state=kept["inputs"], g_state_out=g_inputs_out, g_state=g_inputs, lengths=lengths)
        q, qt = _both(g_s.view(R, 2 * F))
        g_n = torch.empty((R, W), dtype=kept["x_dtype"], device=dev)
        dtst_product(*q, *self.w_in.cols, g_n)
        _weight_gradient(qt, kept["nt"], R, g_w_in)
        g_u, g_norm, g_norm_bias = torch.empty((R, W), dtype=f32, device=dev), torch.empty_like(self.norm), torch.empty_like(self.norm)
        g_x = g_u if kept["x_dtype"] == f32 else torch.empty((R, W), dtype=kept["x_dtype"], device=dev)
        dtst_layer_norm_adj(g_n, kept["u"], self.norm, kept["mean"], kept["rstd"], g_u, g_norm, g_norm_bias,
                            g_sum=None if g_res is None else g_res.reshape(R, W), g_x=None if g_x is g_u else g_x)
        return dict(x=g_x.view(B, T, W), res=g_u.view(B, T, W), state=(g_inputs, g_h), norm=g_norm, norm_bias=g_norm_bias,
                    w_in=g_w_in, b_in=g_s.float().sum(dim=(0, 1)), conv=g_conv, conv_bias=g_conv_bias, w_x=g_w_x,
                    b_x=g_p.float().sum(dim=(0, 1)), a=g_a, d=g_d, w_out=g_w_out)


def clip_gradients(gradients, most, reduce=None):
    """Scales the weights' gradients of the blocks (what their backward returned, a
    list of dicts; x, res and state are left alone) in place so that their norm
    together is at most `most`.  Returns the norm before, one float32 on the device.
    Where other ranks hold other weights' gradients, reduce(square) has to sum one
    float64 in place over them (32 bits do not hold the square of a large norm)."""
    weights = [g for d in gradients for k, g in d.items() if k not in ("x", "res", "state")]
    norm = torch.empty(1, dtype=torch.float32, device=weights[0].device if weights else "cuda")
    dtst_global_norm(weights, norm)
    if reduce is not None:
        square = norm.double().square_()
        reduce(square)
        norm.copy_(square.sqrt_())
    dtst_clip(weights, norm, most)
    return norm


class Rollout:
    """Fields of `channels` channels on one shard, batch sequences at a time.
    grid: a descriptor's n_global, n_local, offset and kmax in x, y, z (3 each);
    blocks: LatentBlocks and SelectiveBlocks of width 2 channels M, M the retained
    modes of one time step (so that 2 channels M is at most 32768).  A shard's
    coefficients are its part of the domain's: where n_local is not n_global,
    reduce(tokens) has to sum them in place over the shards, as
    torch.distributed.all_reduce does; every shard then runs the same blocks on
    the same tokens, and decodes its own part of the field."""

    GROUP = 256  # frames of one plan at most; halved until the library takes such a plan

    def __init__(self, grid, channels, batch, blocks, device="cuda", reduce=None):
        if reduce is None and tuple(grid["n_local"]) != tuple(grid["n_global"]):
            raise ValueError(f"a shard {tuple(grid['n_local'])} of {tuple(grid['n_global'])} holds its part of the "
                             "coefficients: need reduce, which sums them over the shards")
        self.grid, self.channels, self.batch, self.blocks, self.device = grid, channels, batch, list(blocks), device
        self.reduce = reduce
        self.plans = {}
        self.group = self.GROUP
        while self.group > 1 and not self._supported(self.group):
            self.group //= 2
        self.width = 2 * channels * self.plan(1).n_modes
        for b in self.blocks:
            if b.width != self.width:
                raise ValueError(f"a block's width must be 2 * channels * modes = {self.width}")
        self.states = None

    def _desc(self, frames):
        g = self.grid
        return dict(n_global=tuple(g["n_global"]) + (1,), n_local=tuple(g["n_local"]) + (1,),
                    offset=tuple(g["offset"]) + (0,), kmax=tuple(g["kmax"]), kt=1, batch=frames,
                    c_in=self.channels, c_out=self.channels)

    def _supported(self, frames):
        try:
            dtst_desc_validate(self._desc(frames))
        except DtstError as e:
            if e.status != _UNSUPPORTED:
                raise
            return False
        return True

    def plan(self, frames):
        """The plan of `frames` frames at once."""
        if frames not in self.plans:
            self.plans[frames] = Plan(self._desc(frames), self.device)
        return self.plans[frames]

    def _groups(self, frames):
        """Plans and their frames: groups of GROUP frames, then of smaller powers
        of two, so that few plans (each has a workspace) serve any number."""
        i, n = 0, self.group
        while i < frames:
            if n <= frames - i:
                yield self.plan(n), slice(i, i + n)
                i += n
            else:
                n //= 2

    def encode(self, frames):
        """(B, T, channels, x, y, z) float32 to tokens (B, T, width) float32."""
        B, T = frames.shape[:2]
        xhat = torch.empty(B * T, self.width // 2, dtype=torch.complex64, device=self.device)
        flat = frames.contiguous().view(B * T, frames[0, 0].numel() if B * T else 0)
        for plan, s in self._groups(B * T):
            plan.forward(flat[s].view(plan.spatial_shape(self.channels)),
                         xhat[s].view(plan.spectral_shape(self.channels)))
        tokens = torch.view_as_real(xhat).view(B, T, self.width)
        if self.reduce is not None:
            self.reduce(tokens)
        return tokens

    def decode(self, tokens):
        B, T = tokens.shape[:2]
        yhat = torch.view_as_complex(tokens.contiguous().view(B * T, self.width // 2, 2))
        n = self.plan(1).n_local[:3]
        y = torch.empty(B * T, self.channels * n[0] * n[1] * n[2], dtype=torch.float32, device=self.device)
        for plan, s in self._groups(B * T):
            plan.inverse(yhat[s].view(plan.spectral_shape(self.channels)), y[s].view(plan.spatial_shape(self.channels)))
        return y.view(B, T, self.channels, *n)

    def reset(self):
        """Forget the sequences so far."""
        self.states = [b.state(self.batch, self.device) for b in self.blocks]

    def advance(self, frames, lengths=None):
        """The prediction after each of the frames (B, T, channels, x, y, z) of
        the sequences, which go on from the frames of earlier calls."""
        if self.states is None:
            self.reset()
        x, res = self.encode(frames), None
        for block, state in zip(self.blocks, self.states):
            x, res = block.forward(x, res, state, lengths)
        return self.decode(res + x if res is not None else x)

    def march(self, frame, steps):
        """`steps` predictions, each from the one before, after (B, channels, x,
        y, z) and what the sequences have seen."""
        out = torch.empty((frame.shape[0], steps) + tuple(frame.shape[1:]), dtype=torch.float32, device=self.device)
        for t in range(steps):
            frame = self.advance(frame[:, None])[:, 0]
            out[:, t] = frame
        return out

    def close(self):
        for p in self.plans.values():
            p.close()
        self.plans = {}
