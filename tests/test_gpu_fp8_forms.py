"""Every form of the product of 8-bit floating point codes: exact sums, its own streams and graphs."""
import pytest

from fp8_forms import FORMS, whole
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _operand(R, K, fmt, seed):
    import torch
    q, s, v = whole(R, K, seed)
    code = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    return (torch.from_numpy(q).to("cuda:0").to(code), torch.from_numpy(s).to("cuda:0").view(torch.float8_e8m0fnu)), torch.from_numpy(v)


@pytest.mark.parametrize("M,N,K", [f[:3] for f in FORMS])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3")])
def test_exact_sums(M, N, K, fa, fb):
    q8t = require_gpu()
    import torch
    (a, va), (b, vb) = _operand(M, K, fa, 1), _operand(N, K, fb, 2)
    assert 144 * K < 2 ** 24
    want = va @ vb.T
    assert torch.equal(q8t.fp8_gemm(a[0], a[1], b[0], b[1], dtype=torch.float32).cpu(), want)
    assert torch.equal(q8t.fp8_gemm(a[0], a[1], b[0], b[1]).cpu(), want.bfloat16())
