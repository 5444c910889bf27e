"""Norms with infinities and NaN: what they reach and what they do not."""
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _rows(T, D, dtype, seed):
    import torch
    return torch.randn(T, D, generator=torch.Generator().manual_seed(seed)).to(getattr(torch, dtype)).to("cuda:0")


@pytest.mark.parametrize("D", [5, 60, 130, 260, 515, 4100, 8200])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_codes_behind_a_rows_end_are_zeros(D, dtype):
    # rows whose 1 / rms is a NaN (a NaN in the row) or infinite (zeros and eps = 0); the codes are those of y by themselves
    q8t = require_gpu()
    import torch
    x, w = _rows(9, D, dtype, D), torch.ones(D, device="cuda:0")
    x[3] = 0
    x[5, D // 2] = float("nan")
    x[7, 0] = float("inf")
    y, q, s = (q8t.residual_norm_fwd(x, w_pre=w, eps=0.0, quantized=True)[k] for k in (1, 3, 4))
    assert bool(y[3].isnan().all()) and bool(y[5].isnan().all())
    assert not bool(q.view(torch.uint8)[:, D:].any()) and bool(q[5, :D].float().isnan().all())
    if dtype == "float32":
        want = q8t.fp8_quantize(y)
        assert torch.equal(q.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s.view(torch.uint8), want[1].view(torch.uint8))
