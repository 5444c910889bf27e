"""Outputs that the calls make are tensors like any other to those who watch torch make them: dispatch modes, the profiler, deterministic mode."""
import pytest

from gpu_util import require_gpu

pytestmark = pytest.mark.gpu


def _calls(q8t):
    """a call and the number of tensors that it makes"""
    import torch
    x = torch.randn(8, 256, device="cuda:0")
    w = torch.ones(256, device="cuda:0")
    q, s, _, _ = q8t.fp8_quantize(x)
    return [(lambda: q8t.quantize(x), 2), (lambda: q8t.quantize_bifurcate(x), 4), (lambda: q8t.fp8_quantize(x, transposed=True), 4),
            (lambda: q8t.fp8_gemm(q, s, q, s), 1), (lambda: q8t.residual_norm_fwd(x, x, w_pre=w), 3), (lambda: q8t.dropout(x, 0.5), 1)]


def test_a_dispatch_mode_sees_them():
    q8t = require_gpu()
    import torch
    from torch.utils._python_dispatch import TorchDispatchMode

    class Seen(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            out = func(*args, **(kwargs or {}))
            if func.overloadpacket in (torch.ops.aten.empty, torch.ops.aten.empty_like):
                made.append(out.data_ptr())
            return out

    for call, count in _calls(q8t):
        call()                  # scratch memory is kept from here on
        made = []
        with Seen():
            out = call()
        out = [t for t in (out if isinstance(out, tuple) else (out,)) if t is not None]
        assert len(out) == count and sorted(made) == sorted(t.data_ptr() for t in out)


def test_the_profiler_sees_them():
    q8t = require_gpu()
    import torch
    for call, count in _calls(q8t):
        call()
        with torch.autograd.profiler.profile() as p:
            call()
        assert sum(e.name in ("aten::empty", "aten::empty_like") for e in p.function_events) >= count


def test_deterministic_mode_fills_them():
    q8t = require_gpu()
    import torch
    x = torch.randn(8, 256, device="cuda:0")
    calls = _calls(q8t)
    torch.use_deterministic_algorithms(True)
    try:
        for call, _ in calls:
            call()
        stats = q8t.residual_norm_fwd(x, x)[2]      # no norm: its second row is not written
    finally:
        torch.use_deterministic_algorithms(False)
    assert bool((stats[0] == 1).all()) and bool(stats[1].isnan().all())
