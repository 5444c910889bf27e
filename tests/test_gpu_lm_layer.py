"""The operators of the 8-bit layer one after the other, as a residual block uses them: forward, backward, captured, and for one token."""
import numpy as np
import pytest

import lm_layer
import lm_plain as plain
from gpu_util import require_gpu
from lm_layer import BRANCH, EPS, P, RES

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


class Device:
    """The library's calls; check: each against the plain form in 64 bits at its own inputs."""

    def __init__(self, q8t, check, step=None):
        import torch
        self.q8t, self.check, self.step, self.torch = q8t, check, step, torch

    def norm(self, res, h, w_post, gate, w_pre):
        kw = {} if h is None else dict(w_post=w_post, gate=gate, res_scale=RES, branch_scale=BRANCH, p=P, seed=5, step=self.step)
        r, y, st, _, _ = self.q8t.residual_norm_fwd(res, h, w_pre=w_pre, eps=EPS, **kw)
        if r is None:
            r = res
        if self.check:
            H = [plain.host(t) for t in (res, h, w_post, gate, w_pre)]
            keep = None if h is None else plain.kept(h.numel(), P, 5).reshape(h.shape)
            wr, wy, s1, s2 = plain.norm_fwd(*H, EPS, RES, BRANCH, keep)
            # as in the operator's own tests: below 48 roundings of the two terms, 128 of y
            size = np.abs(H[0])
            if h is not None:
                size = np.abs(RES * H[0]) + BRANCH * np.abs(plain.norm_fwd(0 * H[0], *H[1:4], None, EPS, 0.0, 1.0, keep)[0])
            plain.within(r, wr, plain.HALF[r.dtype] * np.abs(wr) + 48 * U * size, "res_out")
            plain.within(y, wy, plain.HALF[y.dtype] * np.abs(wy) + 128 * U * (np.abs(H[4]) * s2[:, None] * size + np.abs(wy)), "y")
        return r, y, st

    def norm_bwd(self, dy, dres_out, r, h, st, w_post, gate, w_pre):
        kw = {} if h is None else dict(w_post=w_post, gate=gate, res_scale=RES, branch_scale=BRANCH, p=P, seed=5, step=self.step)
        got = self.q8t.residual_norm_bwd(dy, dres_out, r, h, st, w_pre=w_pre, **kw)
        if self.check:
            scales = (1.0, 1.0, None) if h is None else (RES, BRANCH, plain.kept(h.numel(), P, 5).reshape(h.shape))
            s = plain.host(st)
            ins = [plain.host(t) for t in (dy, dres_out, r, h)] + [s[0], s[-1]] + [plain.host(t) for t in (w_post, gate, w_pre)]
            want, size = plain.norm_bwd(*ins, *scales), plain.norm_bwd(*ins, *scales, size=True)
            # below 128 roundings over the two norms, and as many additions as rows in the sums over them
            for name, t, w, z in zip(("dres", "dh", "dgate", "dw_post", "dw_pre"), got, want, size):
                if t is not None:
                    rows = dy.shape[0] if name[:2] == "dw" or name == "dgate" else 0
                    plain.within(t, w, plain.HALF[t.dtype] * np.abs(w) + (128 + rows) * U * z, name)
        return got

    def _codes(self, x, fmt, **kw):
        got = self.q8t.fp8_quantize(x, fmt, transposed=True, step=self.step, **kw)
        if self.check:
            r = plain.draws(x.numel(), kw["seed"]).reshape(x.shape) if "seed" in kw else None
            rows = 128 if kw.get("square") else 1
            for q, s, v, rr in ((got[0], got[1], plain.host(x), r), (got[2], got[3], plain.host(x).T, None if r is None else r.T)):
                wq, ws = plain.quantize(v, fmt, rows, rr)
                assert np.array_equal(plain.host(q), wq) and np.array_equal(s.view(self.torch.uint8).cpu().numpy(), ws)
        return got[:2], got[2:]

    def codes(self, x):
        return self._codes(x, "e4m3")

    def weight(self, x):
        return self._codes(x, "e4m3", square=True)

    def gradient(self, x):
        return self._codes(x, "e5m2", stochastic=True, seed=9)

    def product(self, a, b, whole=False):
        got = self.q8t.fp8_gemm(*a, *b, dtype=self.torch.float32 if whole else self.torch.bfloat16)
        if self.check:
            A, B = (plain.values(plain.host(q), s.view(self.torch.uint8).cpu().numpy()) for q, s in (a, b))
            want, size = A @ B.T, np.abs(A) @ np.abs(B).T
            # as in the product's own tests: a partial sum's last place for each addition; bf16: 2^-10 of the matrix instruction, one rounding
            off = A.shape[1] * 2.0 ** -23 * size
            if not whole:
                off = off + 2.0 ** -10 * size
                off = off + 2.0 ** -8 * (np.abs(want) + off)
            plain.within(got, want, off, "product")
        return got

    def drop(self, z):
        got = self.q8t.dropout(z, P, seed=6, step=self.step)
        if self.check:
            want = plain.dropout(plain.host(z), P, 6)
            plain.within(got, want, (plain.HALF[z.dtype] + 2 * U) * np.abs(want), "drop-out")
        return got


def _inputs(T, D, N, groups, dtype):
    import torch
    whole = ("w_in", "w1", "w2", "w_post", "w_pre")          # the parameters stay in fp32
    return {k: torch.from_numpy(v).to(torch.float32 if k in whole else dtype).to("cuda:0") for k, v in lm_layer.inputs(T, D, N, groups).items()}


@pytest.mark.parametrize("T,D,N,groups", [(1, 128, 64, 1), (37, 130, 260, 1), (200, 515, 300, 4), (384, 256, 640, 384), (130, 1025, 1000, 2)])
def test_forward_and_backward(T, D, N, groups):
    q8t = require_gpu()
    import torch
    x = _inputs(T, D, N, groups, torch.bfloat16)
    out, grads = lm_layer.block(Device(q8t, True), x)
    for name, t in {**out, **grads}.items():
        assert bool(torch.isfinite(t.float()).all()), name
    for name, t in grads.items():
        assert t.shape == x[name].shape, name


def test_captured_with_an_eager_block_alive():
    q8t = require_gpu()
    import torch
    x = _inputs(200, 515, 300, 4, torch.bfloat16)
    flat = lambda r: list(r[0].values()) + list(r[1].values())   # noqa: E731
    steps = [torch.tensor([k], device="cuda:0") for k in range(3)]
    want = [flat(lm_layer.block(Device(q8t, False, s), x)) for s in steps]
    assert all(not torch.equal(want[0][k], want[1][k]) for k in range(len(want[0])))   # other masks and other draws
    step = torch.zeros(1, dtype=torch.int64, device="cuda:0")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = flat(lm_layer.block(Device(q8t, False, step), x))
    for k in (0, 2, 1, 0):
        step.copy_(steps[k])
        for t in got:
            t.fill_(7.0)
        graph.replay()
        eager = flat(lm_layer.block(Device(q8t, False, steps[k]), x))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(got, want[k], eager))


@pytest.mark.parametrize("T", [1, 2, 17])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_tokens_to_answers(T, dtype):
    # the form for single tokens: the norm's own codes into the product, no gradients, the whole step as one graph
    q8t = require_gpu()
    import torch
    D, N = 1000, 515
    dt = getattr(torch, dtype)
    x = _inputs(T, D, N, 1, dt)
    q1, s1, t1, u1 = q8t.fp8_quantize(x["w1"], square=True, transposed=True)
    q2, s2, t2, u2 = q8t.fp8_quantize(x["w2"], square=True, transposed=True)

    def step(res):
        _, _, _, q, s = q8t.residual_norm_fwd(res, w_pre=x["w_in"], eps=EPS, quantized=True, want_y=False)
        z = q8t.fp8_gemm(q, s, t1, u1, dtype=dt)
        zq, zs, _, _ = q8t.fp8_quantize(z)
        h = q8t.fp8_gemm(zq, zs, t2, u2, dtype=dt)
        return (q, s, z, zq, zs, h) + tuple(q8t.residual_norm_fwd(res, h, w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], eps=EPS,
                                                                  quantized=True))

    got = step(x["res"])
    v = lambda q, s: plain.values(plain.host(q), s.view(torch.uint8).cpu().numpy())   # noqa: E731
    for y, (a, sa), (b, sb) in ((got[2], got[:2], (t1, u1)), (got[5], got[3:5], (t2, u2))):
        A, B = v(a, sa), v(b, sb)
        want, size = A @ B.T, np.abs(A) @ np.abs(B).T
        off = A.shape[1] * 2.0 ** -23 * size
        if dt == torch.bfloat16:
            off = off + 2.0 ** -10 * size
            off = off + 2.0 ** -8 * (np.abs(want) + off)
        plain.within(y, want, off, "product")
    wq, ws = plain.quantize(plain.host(got[2]), "e4m3")
    assert np.array_equal(plain.host(got[3]), wq) and np.array_equal(got[4].view(torch.uint8).cpu().numpy(), ws)
    y0 = plain.norm_fwd(plain.host(x["res"]), None, None, None, plain.host(x["w_in"]), EPS, 1.0, 1.0, None)[1]
    scale = np.repeat(np.exp2(got[1].view(torch.uint8).cpu().numpy()[:, :8].astype(np.float64) - 127), 128, axis=1)[:, :D]
    # nearest codes: half a step of 2^-3 relative, or of the smallest step; y is off by 128 roundings before
    assert (np.abs(v(*got[:2])[:, :D] - y0) <= 2.0 ** -4 * np.abs(y0) * (1 + 1e-4) + scale * 2.0 ** -10 * (1 + 1e-4) + 256 * U * np.abs(y0)).all()
    graph = torch.cuda.CUDAGraph()
    res = x["res"].clone()
    with torch.cuda.graph(graph):
        again = step(res)
    for sign in (1.0, -0.5, 1.0):
        res.copy_(x["res"] * sign)
        graph.replay()
        eager = step(x["res"] * sign)
        torch.cuda.synchronize()
        assert all((a is None and b is None) or torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(again, eager))


def test_outputs_are_ordinary_tensors():
    # in and out of inference mode, with the storage of a tensor that torch makes
    q8t = require_gpu()
    import torch
    x = _inputs(6, 256, 64, 1, torch.bfloat16)

    def outputs():
        return [t for t in q8t.residual_norm_fwd(x["res"], x["res"], w_pre=x["w_pre"], quantized=True) if t is not None] + \
            [t for t in q8t.fp8_quantize(x["w1"], transposed=True)] + [q8t.dropout(x["res"], 0.5)]

    for t in outputs():
        assert not t.is_inference() and t.is_contiguous() and t.storage_offset() == 0 and t.untyped_storage().nbytes() >= t.numel() * t.element_size()
    y = outputs()[1]
    y.requires_grad_(True)
    (y.float() * 2).sum().backward()
    assert torch.equal(y.grad.float(), torch.full_like(y.float(), 2.0))
    with torch.inference_mode():
        assert all(t.is_inference() for t in outputs())
        z = outputs()[-1].add_(1)
    assert z.shape == x["res"].shape
