"""Whose memory a call's result and workspace are, without a GPU: what the binding asks of
torch's allocator."""
import pytest

swan = pytest.importorskip("paper_2511_18936_amd.swan")


class _Block:
    is_cuda, device = True, "cuda:0"

    def __init__(self, how, stream):
        self.how, self.stream, self.kept_for = how, stream, []

    def record_stream(self, stream):
        self.kept_for.append(stream)


@pytest.mark.parametrize("how", ["empty", "zeros"])
def test_a_result_is_kept_for_the_current_stream(monkeypatch, how):
    """Made for the call's stream; where another one is current, which the caller may use it
    on, dropping it waits for that one's work."""
    import torch

    monkeypatch.setattr(swan, "_made", lambda how, shape, dtype, device, stream: _Block(how, stream))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "current")
    t = swan._result(how, (3,), "uint8", "cuda:0", "side")
    assert (t.how, t.stream, t.kept_for) == (how, "side", ["current"])
    assert swan._result(how, (3,), "uint8", "cuda:0", "current").kept_for == []
    assert swan._result(how, (3,), "uint8", "cuda:0", None).kept_for == []
