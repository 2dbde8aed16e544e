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


@pytest.mark.parametrize("call", ["calibrate_rotation", "calibrate_rotations", "change_k", "rope"])
def test_other_calls_make_their_memory_on_their_stream(monkeypatch, call):
    """Workspaces, cleared pages and results of the calls that are not decode steps."""
    import torch

    cache, made = _cache(), []

    class Stream:
        cuda_stream = 0

        def synchronize(self):
            pass

    side = Stream()

    def make(how, shape, dtype, device, stream):
        made.append(stream)
        dtype = getattr(torch, dtype) if isinstance(dtype, str) else dtype
        return getattr(torch, how)(shape, dtype=dtype)

    class Lib:
        def __getattr__(self, name):
            return (lambda *args: 0) if name != "swan_calibrate_workspace_bytes" and \
                name != "swan_cache_bytes" else getattr(real, name)

    real = swan._lib
    monkeypatch.setattr(swan, "_made", make)
    monkeypatch.setattr(swan, "_lib", Lib())
    monkeypatch.setattr(swan, "_on_gpu", lambda **tensors: None)
    rows, P = torch.zeros(300, 128), torch.zeros(2, 128, 128)
    if call == "calibrate_rotation":
        swan.calibrate_rotation(rows, P[0], stream=side)
    elif call == "calibrate_rotations":
        swan.calibrate_rotations(rows, [100, 200], P, stream=side)
    elif call == "change_k":
        cache.change_k([32, 64], stream=side)
    else:
        swan.rope(torch.zeros(2, 1, 3, 128), [0, 5], 10000.0, stream=side)
    assert made and all(s is side for s in made)
