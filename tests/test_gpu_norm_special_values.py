"""Norms with infinities and NaN: what they reach and what they do not."""
import pytest

import lm_plain as plain
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


@pytest.mark.parametrize("T,D", [(6, 5), (40, 100), (23, 515), (12, 4096), (9, 5119), (6, 8200)])
@pytest.mark.parametrize("groups", [1, 2, "T"])
@pytest.mark.parametrize("dtype,dres", [("float32", True), ("bfloat16", True), ("bfloat16", False)])
def test_dropped_positions_give_nothing_to_the_gradients(T, D, groups, dtype, dres):
    # h and a gate a token are not a number where they are dropped: the forward pass does not see it, and so does no gradient
    q8t = require_gpu()
    import torch
    if groups == 2 and T % 2:
        groups = 1
    x = {k: _rows(T, D, dtype, i) for i, k in enumerate(("res", "h", "dy", "dres"))}
    gate = _rows(T if groups == "T" else groups, D, dtype, 9)
    w = 1.0 + _rows(1, D, "float32", 10)[0]
    keep = torch.from_numpy(plain.kept(T * D, 0.5, 3).reshape(T, D) != 0).to("cuda:0")

    def both():
        r, y, st, _, _ = q8t.residual_norm_fwd(x["res"], x["h"], gate=gate, w_pre=w, p=0.5, seed=3)
        return (r, y) + q8t.residual_norm_bwd(x["dy"], x["dres"] if dres else None, r, x["h"], st, gate=gate, w_pre=w, p=0.5, seed=3)[:3]

    want = both()
    x["h"][~keep] = float("nan")
    x["h"].view(-1)[(~keep).view(-1).nonzero()[::2, 0]] = float("inf")
    if groups == "T":
        gate[~keep] = float("nan")
    assert all(torch.equal(a, b) for a, b in zip(both(), want))


def test_nothing_kept_gives_no_gradient():
    q8t = require_gpu()
    import torch
    x = {k: _rows(7, 130, "float32", i) for i, k in enumerate(("res", "dy"))}
    h, gate, w = torch.full((7, 130), float("nan"), device="cuda:0"), torch.ones(1, 130, device="cuda:0"), torch.ones(130, device="cuda:0")
    r, _, st, _, _ = q8t.residual_norm_fwd(x["res"], h, gate=gate, w_pre=w, p=1.0)
    _, dh, dgate, _, _ = q8t.residual_norm_bwd(x["dy"], None, r, h, st, gate=gate, w_pre=w, p=1.0)
    assert torch.equal(r, x["res"]) and not bool(dh.any()) and not bool(dgate.any())
