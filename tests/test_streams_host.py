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


def _cache():
    import torch

    cache = swan.SwanCache(2, 4, 2, 16, 4096, [64, 64], torch.float16, "cpu")
    cache.seq_len = [500, 20]
    return cache


def test_workspaces_of_a_cache_share_no_memory():
    cache = _cache()
    a, b = cache.workspace(), cache.workspace()
    assert a.numel() == b.numel() >= 1 and a.data_ptr() != b.data_ptr()
    small = cache.workspace([1, 1])
    assert small.numel() < a.numel() < cache.workspace([4000, 4000]).numel()


@pytest.mark.parametrize("call", ["decode", "step"])
def test_a_call_has_a_workspace_of_its_own_stream(monkeypatch, call):
    """decode() and step() take a workspace each, made for the stream that the call is on,
    also when the plan grows."""
    import torch

    cache, made, used = _cache(), [], []
    empty = torch.empty(0, dtype=torch.uint8)
    monkeypatch.setattr(swan, "_made", lambda how, shape, dtype, device, stream:
                        made.append((shape[0], stream)) or empty.new_empty(shape))
    at = {"decode": 7, "step": 9}[call]
    monkeypatch.setattr(swan, "decode_attention" if call == "decode" else "decode_step",
                        lambda *args: used.append(args))
    q = torch.zeros(2, 4, 128, dtype=torch.float16)
    k = torch.zeros(2, 2, 1, 128, dtype=torch.float16)
    for i in range(3):
        cache.seq_len = [500 + 1000 * i, 20]
        if call == "decode":
            cache.decode(q, None, None, out=q, stream="side")
        else:
            cache.step(k, k, q, None, None, out=q, stream="side")
    assert [stream for _, stream in made] == ["side"] * 3
    spaces = [args[at] for args in used]
    assert [t.numel() for t in spaces] == [n for n, _ in made]
    assert len({t.data_ptr() for t in spaces}) == 3 and spaces[0].numel() < spaces[2].numel()
    assert all("side" in args for args in used)
