"""What the binding and the library of the latent-sequence operators settle on
the host, without a GPU."""

import contextlib

import pytest
import torch

from test_seq_oracle_cpu import P, recur_call

D = pytest.importorskip("paper_2607_14394_amd", reason="libdtst.so not built")


@pytest.mark.parametrize("stream,pool", [(None, 5), (5, 5), (9, 9), (0, 0)])
def test_a_workspace_comes_from_the_memory_of_the_calls_stream(monkeypatch, stream, pool):
    """On another stream's memory a block may still be in use by what that
    stream has queued."""
    current, taken, empty = [5], [], torch.empty

    @contextlib.contextmanager
    def on(s):
        current.append(s)
        yield
        current.pop()

    def record(*a, **kw):
        taken.append(current[-1])
        return empty(*a, **kw)

    monkeypatch.setattr(D, "torch_stream", lambda: current[-1])
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda s, device=None: s)
    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, s: None)
    monkeypatch.setattr(torch, "empty", record)
    p, n, ws = D._scratch(None, 100, torch.device("cpu"), stream)
    assert taken == [pool] and n == 100 and p == ws.data_ptr() and current == [5]


def test_a_rollout_on_a_shard_needs_the_sum_over_the_shards():
    from paper_2607_14394_amd.rollout import Rollout
    for local, offset in (((4, 8, 8), (4, 0, 0)), ((8, 8, 7), (0, 0, 0))):
        with pytest.raises(ValueError, match="reduce"):
            Rollout(dict(n_global=(8, 8, 8), n_local=local, offset=offset, kmax=(1, 1, 1)), 1, 1, [], device="cpu")


# batch 2, steps 300, features 16: entries 4800 elements apart, steps 16; h: 128
# bytes, states: 384, the workspace 6208
@pytest.mark.parametrize("kw,word", [
    (dict(h=P), "z and h_out"), (dict(h=P * 2 + 9600 * 2 - 4), "v and h_out"), (dict(h=P * 3 - 124), "o and h_out"),
    (dict(h=P * 4 + 4), "y and h_out"), (dict(h0=P * 4), "y and h_zero"), (dict(h0=P * 5, h=P * 5 + 64), "h_out and h_zero"),
    (dict(n=P * 4 + 8), "y and lengths"), (dict(n=P * 5, h=P * 5 - 124), "h_out and lengths"),
    (dict(st=P), "z and states"), (dict(st=P * 5, h0=P * 5 + 380), "states and h_zero"),
    (dict(st=P * 5, h=P * 5 - 64), "states and h_out"), (dict(st=P * 5, n=P * 5 + 380), "states and lengths"),
    (dict(st=P * 4), "y and states"), (dict(ws=P * 2), "v and workspace"), (dict(ws=P * 4), "y and workspace"),
    (dict(ws=P * 8, st=P * 8 + 6204), "workspace and states"), (dict(h=P * 8), "workspace and h_out"),
    (dict(h0=P * 8 + 128), "workspace and h_zero"), (dict(n=P * 8), "workspace and lengths"),
])
def test_recurrence_refuses_shared_states(kw, word):
    st, msg = recur_call(**kw)
    assert st == 1 and msg == word + " overlap", msg


# (h0 stands for g_h and h for g_hzero here, y for g_y)
@pytest.mark.parametrize("kw,word", [
    (dict(h=P), "z and g_hzero"), (dict(h=P * 4), "g_y and g_hzero"), (dict(h=P * 6 + 19196), "g_v and g_hzero"),
    (dict(h=P * 9), "g_hzero and states"), (dict(h0=P * 10, h=P * 10 + 64), "g_hzero and g_h"),
    (dict(h0=P * 5), "g_z and g_h"), (dict(st=P * 7), "g_o and states"), (dict(n=P * 5), "g_z and lengths"),
    (dict(n=P * 10, h=P * 10 - 124), "g_hzero and lengths"), (dict(ws=P), "z and workspace"),
    (dict(ws=P * 6), "g_v and workspace"), (dict(ws=P * 9 - 6192), "workspace and states"),
    (dict(h0=P * 8), "workspace and g_h"), (dict(h=P * 8), "workspace and g_hzero"), (dict(n=P * 8), "workspace and lengths"),
])
def test_recurrence_adj_refuses_shared_states(kw, word):
    st, msg = recur_call(fn="dtst_recurrence_adj", **dict(dict(st=P * 9), **kw))
    assert st == 1 and msg == word + " overlap", msg


def test_a_rollout_keeps_few_plans(monkeypatch):
    from paper_2607_14394_amd import rollout
    made = []

    class Counted:
        n_modes = 8

        def __init__(self, desc, device):
            made.append(desc["batch"])

    monkeypatch.setattr(rollout, "Plan", Counted)
    ro = rollout.Rollout(dict(n_global=(8, 8, 8), n_local=(8, 8, 8), offset=(0, 0, 0), kmax=(1, 1, 1)), 1, 1, [], device="cpu")
    for frames in range(700):
        at = 0
        for _, s in ro._groups(frames):
            assert s.start == at and s.stop > at
            at = s.stop
        assert at == frames
    assert len(made) == len(set(made)) <= 9 and max(made) == ro.group


def test_a_block_wider_than_the_norm_is_refused_when_it_is_made():
    from paper_2607_14394_amd.rollout import LatentBlock
    W, F = 32769, 1
    meta = lambda *s: torch.empty(s, device="meta")  # noqa: E731
    with pytest.raises(ValueError, match="width 32769.*32768"):
        LatentBlock(meta(W), meta(3 * F, W), meta(3 * F), meta(W, F))
    with pytest.raises(ValueError, match="width 0"):
        LatentBlock(meta(0), meta(3, 0), meta(3), meta(0, 1))
