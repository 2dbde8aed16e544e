"""Layers behind another one's tokens, without a GPU: which positions and which project()
they have."""
import types

import pytest

swan = pytest.importorskip("paper_2511_18936_amd.swan")

from paper_2511_18936_amd.layer import SwanAttentionLayer  # noqa: E402


class _Own(SwanAttentionLayer):
    def project(self, x):
        return self.positions(), x, x


def _layer(cls=SwanAttentionLayer):
    import torch

    layer = cls.__new__(cls)
    layer.n_heads = layer.n_kv_heads = 1
    layer.dtype = torch.float16
    layer.P_qk = "P_qk"
    layer.cache = swan.SwanCache(2, 1, 1, 4, 100, [8, 8], torch.float16, "cpu")
    layer.cache.seq_len = [30, 40]
    return layer


def _fork(layer, of=(0, 1, 1)):
    return layer.fork(list(of), 4, 50, [8] * len(of))


def _with(method):
    """A layer whose project() was replaced on the object: by a method of it, or a function."""
    layer = _layer()
    layer.project = types.MethodType(lambda self, x: (self.positions(), x, x), layer) if method \
        else (lambda x: (layer.positions(), x, x))
    return layer


@pytest.mark.parametrize("make", [lambda: _layer(_Own), lambda: _with(True)])
def test_an_own_project_asks_the_fork_for_positions(make):
    layer = make()
    fork = _fork(layer)
    assert fork.project(None)[0] == [30, 40, 40]
    fork.cache.seq_len = [1, 2, 3]
    assert fork.project(None)[0] == [31, 42, 43]
    assert layer.project(None)[0] == [30, 40]


@pytest.mark.parametrize("n,attend", [(1, False), (5, False), (5, True)])
def test_a_function_of_the_parent_is_not_used_for_the_fork(n, attend):
    """It may rotate to the parent's positions: refused until the fork has its own."""
    import torch

    layer = _with(False)
    fork = _fork(layer)
    x = torch.zeros(3, n, 4)
    with pytest.raises(ValueError, match="project"):
        fork(x, attend=attend)
    assert fork.cache.seq_len == [0, 0, 0] and layer.project(None)[0] == [30, 40]
    fork.project = lambda x: (fork.positions(), x, x)
    assert fork.project(None)[0] == [30, 40, 40]


@pytest.mark.parametrize("own", [False, True])
@pytest.mark.parametrize("n,attend", [(1, False), (5, False), (5, True)])
def test_a_parent_that_grows_is_refused(n, attend, own):
    """Positions behind it would move; sequences that no fork stands behind may grow."""
    import torch

    layer = _layer()
    fork = _fork(layer, [1, 1, 1])
    if own:
        fork.project = lambda x: (x, x, x)
    layer.cache.seq_len = [31, 40]
    assert fork.positions() == [40, 40, 40]
    layer.cache.seq_len = [31, 41]
    with pytest.raises(ValueError, match="grown"):
        fork.positions()
    with pytest.raises(ValueError, match="grown"):
        fork(torch.zeros(3, n, 4), attend=attend)
    assert fork.cache.seq_len == [0, 0, 0]
