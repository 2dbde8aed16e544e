"""swan_qkv_rows with every eps that it takes, finite and not negative."""
import numpy as np
import pytest

from tests.test_gpu_qkv_rows import _close, _formula, _make

pytestmark = pytest.mark.gpu
D = 128
EPS = [0.0, 5e-324, 1e-310, 1e-300, 1e-60, 1e-45, 1e-42, 1e-39, 1e-38, 1e-12, 1.0, 1e30, 1e38, 1e39,
       1e60]


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("name", ["float16", "float32"])
@pytest.mark.parametrize("n", [3, 900])  # a wave per row, 4 positions a workgroup
def test_any_eps(gpu_device, swan_mod, torch_mod, n, name, eps):
    """Rows of zeros stay zeros for any eps above 0 and are no numbers for 0, 0 times an
    infinity; all others are the formula, with weights as large as 1 / sqrt(eps) is small."""
    torch = torch_mod
    dtype = getattr(torch, name)
    x = _make(torch, gpu_device, 2, n, 4, 2, dtype, n)
    x[0, 1, :2 * D] = 0
    x[1, n - 1] = 0
    x[0, 2] = x[0, 2] * 2.0 ** -13  # the smallest ones of their type among them
    big = min(max(1.0, eps) ** 0.5, 1e30)
    g = torch.Generator().manual_seed(9)
    w = ((1 + 0.3 * torch.randn(D, generator=g)) * big).to(gpu_device)
    got = swan_mod.qkv_rows(x, 4, 2, [3, 70000], 10000.0, w, w, eps=eps)
    host = w.double().cpu().numpy()
    with np.errstate(divide="ignore", invalid="ignore"):
        want = _formula(x.double().cpu().numpy(), 4, 2, [3, 70000], 10000.0, host, host, eps)
    for part, (a, b) in enumerate(zip(got, want)):
        nan = np.isnan(b)
        assert np.array_equal(np.isnan(a.double().cpu().numpy()), nan), part
        assert nan.any() == (eps == 0 and part < 2)
        clean = torch.where(torch.tensor(nan, device=gpu_device), torch.zeros_like(a), a)
        _close(clean, np.where(nan, 0.0, b), dtype)
        zero = (x.view(2, n, 8, D)[:, :, (0, 4, 6)[part]:(4, 6, 8)[part]] == 0).all(-1)
        if eps:
            assert (a.transpose(1, 2)[zero] == 0).all()
