"""The plan of a windowed decode call is its own: swan_set_decode_tuning, which is for the calls
without a window, does not change it (on the CPU: the workspaces that plans ask for)."""
import pytest
import torch

from paper_2511_18936_amd import swan


@pytest.fixture
def tuned():
    yield lambda: swan.set_decode_tuning(target_waves=64, short_split_pages=-1, merge_pct=-1,
                                         side_streams=-1)
    swan.set_decode_tuning()


@pytest.mark.parametrize("hq,hkv", [(8, 8), (32, 8)])
def test_a_window_is_planned_apart(tuned, hq, hkv):
    cache = swan.SwanCache(3, hq, hkv, 64, 8192, [64, 48, 96], torch.float16, "cpu")
    lens = [8000, 4000, 700]
    ask = lambda: swan.decode_window_workspace_bytes(cache.desc, lens, cache.k_active, 4096, 4)  # noqa: E731
    plain = lambda: swan.decode_workspace_bytes(cache.desc, lens, cache.k_active)  # noqa: E731
    before = ask(), plain()
    tuned()
    assert ask() == before[0] and plain() < before[1]
