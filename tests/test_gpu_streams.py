"""Calls on a stream that is not the current one: whose memory their results and workspaces
are, and when it is used again."""
import pytest

from tests import rows_ref as R

pytestmark = pytest.mark.gpu
D = 128


def _busy(torch, device):
    """Work of some milliseconds on the current stream."""
    a = torch.ones(4096, 4096, device=device)
    for _ in range(20):
        a = a @ a * 2.0 ** -12
    return a


def _caches(swan_mod, gpu_device):
    own, P_qk, P_vo = R.filled_cache(swan_mod, gpu_device, [300, 40, 500], 8, 2, 16, [64] * 3, "f16",
                                     71)
    past, _, _ = R.filled_cache(swan_mod, gpu_device, [900], 8, 2, 16, [64], "f16", 72,
                                P=(P_qk, P_vo))
    return own, past, P_qk, P_vo


@pytest.mark.parametrize("call", ["decode", "decode prefix", "step", "attend", "prompt", "rows"])
def test_a_result_used_on_the_current_stream_and_dropped(gpu_device, swan_mod, torch_mod, call):
    """Its memory is not given to the call's stream again while the current one reads it."""
    torch = torch_mod
    own, past, P_qk, P_vo = _caches(swan_mod, gpu_device)
    g = torch.Generator().manual_seed(1)
    rows = torch.randn(3, 8, 1, D, generator=g).half().to(gpu_device)
    kv = torch.randn(3, 2, 1, D, generator=g).half().to(gpu_device)
    q = rows[:, :, 0].contiguous()
    qkv = torch.randn(3, 1, 12 * D, generator=g).half().to(gpu_device)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    run = {"decode": lambda: own.decode(q, P_qk, P_vo, stream=side),
           "decode prefix": lambda: own.decode(q, P_qk, P_vo, stream=side,
                                               prefix=swan_mod.Prefix(past)),
           "step": lambda: own.step(kv, kv, q, P_qk, P_vo, stream=side),
           "attend": lambda: own.attend(rows, P_qk, P_vo, stream=side)[0],
           "prompt": lambda: swan_mod.prompt_attention(rows, kv, kv, stream=side),
           "rows": lambda: swan_mod.qkv_rows(qkv, 8, 2, [0] * 3, 10000.0, stream=side)[0]}[call]
    result = run()
    side.synchronize()
    want = result.clone()
    torch.cuda.synchronize()
    keep = _busy(torch, gpu_device)
    kept = result.clone()  # behind the work above
    place, shape = result.data_ptr(), result.shape
    del result
    with torch.cuda.stream(side):
        others = [torch.full(shape, 7.0, dtype=want.dtype, device=gpu_device) for _ in range(50)]
    busy = not torch.cuda.current_stream().query()
    torch.cuda.synchronize()
    assert busy, "the current stream was done too early to show anything"
    assert all(t.data_ptr() != place for t in others)
    assert torch.equal(kept, want)
    del keep
