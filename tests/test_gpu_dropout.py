"""Drop-out with a drawn mask: against the plain form in 64 bits (lm_plain.py)."""
import numpy as np
import pytest

import lm_plain as plain
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _data(n, dtype, seed=0):
    import torch
    return torch.randn(n, generator=torch.Generator().manual_seed(seed)).to(dtype).to("cuda:0")


@pytest.mark.parametrize("n", [0, 1, 3, 7, 8, 9, 2047, 2048, 2049, 100003])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 1.0])
def test_against_plain(n, dtype, p):
    q8t = require_gpu()
    import torch
    dt = getattr(torch, dtype)
    x, r = _data(n, dt, 1), _data(n, dt, 2)
    seed = 0xFEDCBA9876543210
    step = torch.tensor([5], device="cuda:0")
    # a product and, with the residual, a sum: one rounding each in fp32, then one to the type
    for res in (None, r):
        got = q8t.dropout(x, p, seed=seed, step=step, residual=res)
        hx, hr = plain.host(x), plain.host(res)
        want = plain.dropout(hx, p, seed + 5, hr)
        off = plain.HALF[dt] * np.abs(want) + 2.0 ** -23 * (np.abs(hx) / max(1 - p, 0.5) + (0 if res is None else np.abs(hr)))
        plain.within(got, want, off, (n, dtype, p))
        assert got.dtype == dt
    if n and p in (0.1, 0.5):   # kept positions are exactly those of the generator
        one = torch.ones(n, device="cuda:0")
        assert np.array_equal(plain.host(q8t.dropout(one, p, seed=seed)) != 0, plain.kept(n, p, seed) != 0)


@pytest.mark.parametrize("off", [0, 1, 3])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_views_at_any_offset_and_in_place(off, dtype):
    q8t = require_gpu()
    import torch
    n = 5001
    buf = _data(n + off + 9, getattr(torch, dtype), 3)
    x = buf[off:off + n]
    want = q8t.dropout(x.clone(), 0.3, seed=9, residual=x.clone())
    behind = buf[off + n:].clone()
    got = q8t.dropout(x, 0.3, seed=9, residual=x, out=x)
    assert got.data_ptr() == x.data_ptr() and torch.equal(x, want) and torch.equal(buf[off + n:], behind)


def test_values_that_are_dropped_have_no_effect():
    q8t = require_gpu()
    import torch
    n, p = 4096, 0.5
    keep = plain.kept(n, p, 77) != 0
    x = torch.randn(n, device="cuda:0")
    dropped = torch.from_numpy(~keep).to("cuda:0")
    bad = x.clone()
    bad[dropped] = float("nan")
    bad[dropped.nonzero()[::2, 0]] = float("inf")
    assert torch.equal(q8t.dropout(bad, p, seed=77), q8t.dropout(x, p, seed=77))
    x[torch.from_numpy(keep).to("cuda:0").nonzero()[0, 0]] = float("nan")
    assert int(q8t.dropout(x, p, seed=77).isnan().sum()) == 1


def test_backward_is_the_same_call():
    q8t = require_gpu()
    import torch
    x, g = torch.randn(999, device="cuda:0"), torch.randn(999, device="cuda:0")
    y, dx = q8t.dropout(x, 0.2, seed=4), q8t.dropout(g, 0.2, seed=4)
    # <dy, f(x)> = <f'(dy), x>: the operation is linear and its matrix diagonal
    a, b = float((y.double() * g.double()).sum()), float((dx.double() * x.double()).sum())
    assert abs(a - b) <= 2.0 ** -22 * float((y.double() * g.double()).abs().sum())


def test_beyond_32_bits():
    q8t = require_gpu()
    import torch
    n = 2 ** 31 + 12345
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda:0")
    y = q8t.dropout(x, 0.25, seed=11)
    for start in (0, 2 ** 31 - 8, n - 77):
        i = np.arange(start, min(start + 500, n))
        h = np.array([_r16(int(k), 11) for k in i])
        assert np.array_equal(plain.host(y[start:start + len(i)]) != 0, h >= 16384)


def _r16(i, seed):
    import oracle
    return oracle.r16(i, seed)


def test_captured_call_draws_anew_with_its_counter():
    q8t = require_gpu()
    import torch
    x = torch.randn(3000, device="cuda:0")
    step = torch.zeros(1, dtype=torch.int64, device="cuda:0")
    q8t.dropout(x, 0.4, seed=8, step=step)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = q8t.dropout(x, 0.4, seed=8, step=step)
        step.add_(1)
    step.zero_()
    for k in range(4):
        graph.replay()
        eager = q8t.dropout(x, 0.4, seed=8 + k)
        torch.cuda.synchronize()
        assert torch.equal(y, eager)


def test_refusals():
    q8t = require_gpu()
    import torch
    x = torch.zeros(8, 8, device="cuda:0")
    for call in (lambda: q8t.dropout(x.half(), 0.1), lambda: q8t.dropout(x.t()[:4], 0.1), lambda: q8t.dropout(x, 0.1, residual=x[:4]),
                 lambda: q8t.dropout(x, 0.1, residual=x.bfloat16()), lambda: q8t.dropout(x, 0.1, out=x.bfloat16()),
                 lambda: q8t.dropout(x, 0.1, step=torch.zeros(1, device="cuda:0")), lambda: q8t.dropout(x, 0.1, residual=x.cpu())):
        with pytest.raises(ValueError):
            call()
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(q8t.Q8TError):
            q8t.dropout(x, p)
