"""What the binding and the library of the latent-sequence operators settle on
the host, without a GPU."""

import contextlib

import pytest
import torch

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
