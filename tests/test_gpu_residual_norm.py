"""Norms behind and in front of a block with its gate and residual scale: against the plain form in 64 bits (lm_plain.py)."""
import numpy as np
import pytest

import lm_plain as plain
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SHAPES = [(1, 1), (1, 7), (2, 8), (5, 63), (4, 64), (7, 130), (9, 512), (6, 513), (3, 1000), (12, 1024), (10, 2047), (4, 2048), (6, 4096), (3, 4100),
          (2, 5120), (3, 8192), (2, 8193), (2, 16384), (600, 65), (1025, 256)]


def _t(shape, seed, dtype, scale=1.0, add=0.0):
    import torch
    t = torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale + add
    return t.to(dtype).to("cuda:0")


def _inputs(T, D, dtype, post, groups, seed=0):
    import torch
    dt = getattr(torch, dtype)
    s = 100 * seed
    return dict(res=_t((T, D), s + 1, dt, 2.0), h=_t((T, D), s + 2, dt), w_post=_t((D,), s + 3, torch.float32, 0.3, 1.0) if post else None,
                gate=_t((groups, D), s + 4, dt, 0.5, 0.5) if groups else None, w_pre=_t((D,), s + 5, torch.float32, 0.3, 1.0),
                dy=_t((T, D), s + 6, dt), dres_out=_t((T, D), s + 7, dt))


def _check_fwd(q8t, x, p, rs=0.9, bs=0.6, seed=123, eps=1e-5):
    import torch
    step = torch.tensor([7], device="cuda:0")
    T, D = x["res"].shape
    dt = x["res"].dtype
    out = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], eps=eps, res_scale=rs, branch_scale=bs,
                                p=p, seed=seed, step=step, quantized=True)
    H = {k: plain.host(v) for k, v in x.items()}
    keep = plain.kept(T * D, p, seed + 7).reshape(T, D) if p else np.ones((T, D))
    args = (H["w_post"], H["gate"], H["w_pre"])
    r, y, s1, s2 = plain.norm_fwd(H["res"], H["h"], *args, eps, rs, bs, keep)
    # 1/rms: squares, up to 16 + 6 + 16 additions, mean, eps, root and quotient: 24 roundings of a positive sum halved by the root
    plain.within(out[2], np.stack([s1, s2]), 32 * U * np.stack([s1, s2]) + 64 * U * s2 * np.array([[0.0], [1.0]]), "stats")
    # scalars in fp32, 1/rms, a product for each factor and the sum: below 48 roundings of the two terms
    branch = bs * np.abs(plain.norm_fwd(H["res"] * 0, H["h"], H["w_post"], H["gate"], None, eps, 0.0, 1.0, keep)[0])
    size = np.abs(H["res"] * rs) + branch
    plain.within(out[0], r, plain.HALF[dt] * np.abs(r) + 48 * U * size, "res_out")
    ysize = np.abs(H["w_pre"]) * s2[:, None] * size
    plain.within(out[1], y, plain.HALF[dt] * np.abs(y) + 128 * U * (ysize + np.abs(y)), "y")
    # codes: of a y that is off by as much, so a step of the format more where that crosses a border between two codes
    q, s = out[3], out[4].view(torch.uint8).cpu().numpy()
    wq, ws = plain.quantize(y, "e4m3")
    nb = -(-D // 128)
    assert (s[:, nb:] == 127).all() and not plain.host(q)[:, D:].any()
    got = plain.values(plain.host(q), s)[:, :D]
    scale = np.repeat(np.exp2(s[:, :nb].astype(np.float64) - 127), 128, axis=1)[:, :D]
    assert (np.abs(got - y) <= 2.0 ** -4 * np.abs(y) * (1 + 1e-4) + scale * 2.0 ** -10 * (1 + 1e-4) + 128 * U * (ysize + np.abs(y))).all()
    assert (np.abs(s.astype(int) - ws) <= 1).all() and (s != ws).mean() < 0.01 + 1.0 / s.size
    return out


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("post,gated,p", [(True, 1, 0.0), (True, 0, 0.3), (False, 2, 0.0), (False, 0, 0.0), (True, 2, 0.1)])
def test_forward(T, D, dtype, post, gated, p):
    q8t = require_gpu()
    groups = {0: 0, 1: 1, 2: T}[gated]
    _check_fwd(q8t, _inputs(T, D, dtype, post, groups), p)


def _check_bwd(q8t, x, p, parts=("dy", "dres_out"), rs=0.9, bs=0.6, seed=55):
    T, D = x["res"].shape
    dt = x["res"].dtype
    H = {k: plain.host(v) for k, v in x.items()}
    keep = plain.kept(T * D, p, seed).reshape(T, D) if p else np.ones((T, D))
    w_pre = x["w_pre"] if "dy" in parts else None
    fwd = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=w_pre, res_scale=rs, branch_scale=bs, p=p, seed=seed)
    dro = x["dres_out"] if "dres_out" in parts else None
    got = q8t.residual_norm_bwd(x["dy"] if "dy" in parts else None, dro, fwd[0], x["h"], fwd[2], w_post=x["w_post"], gate=x["gate"], w_pre=w_pre,
                                res_scale=rs, branch_scale=bs, p=p, seed=seed)
    s = plain.host(fwd[2])
    ins = (H["dy"], H["dres_out"] if dro is not None else None, plain.host(fwd[0]), H["h"], s[0], s[1], H["w_post"], H["gate"],
           H["w_pre"] if w_pre is not None else None, rs, bs, keep)
    want, size = plain.norm_bwd(*ins), plain.norm_bwd(*ins, size=True)
    # a row's means: 8 to 16 terms a thread, then 22 additions; below 128 roundings over the two norms.  Sums over T rows: T more.
    for name, g, w, z in zip(("dres", "dh", "dgate", "dw_post", "dw_pre"), got, want, size):
        assert (g is None) == (w is None), name
        if g is None:
            continue
        assert g.dtype == (dt if name[:3] != "dw_" else s_type())
        rows = T if name.startswith("dw") or name == "dgate" else 0
        plain.within(g, w, plain.HALF[g.dtype] * np.abs(w) + (128 + rows) * U * z, name)
    return got


def s_type():
    import torch
    return torch.float32


@pytest.mark.parametrize("T,D", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("post,gated,p", [(True, 1, 0.0), (True, 0, 0.3), (False, 2, 0.0), (False, 0, 0.0), (True, 2, 0.1), (False, 1, 0.1)])
def test_backward(T, D, dtype, post, gated, p):
    q8t = require_gpu()
    _check_bwd(q8t, _inputs(T, D, dtype, post, {0: 0, 1: 1, 2: T}[gated]), p)


@pytest.mark.parametrize("T,groups", [(6, 2), (6, 3), (1000, 4), (1000, 125), (1500, 500), (1026, 513), (2000, 2), (1200, 600), (1201, 1201), (4000, 1)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_shared_gates(T, groups, dtype):
    # groups shorter and longer than the rows that one workgroup takes
    q8t = require_gpu()
    x = _inputs(T, 136, dtype, True, groups)
    _check_fwd(q8t, x, 0.0)
    _check_bwd(q8t, x, 0.2)


@pytest.mark.parametrize("T,D,groups", [(1, 64, 1), (2, 100, 2), (3, 128, 1), (3, 256, 3), (5, 9, 5), (1001, 64, 7), (1001, 100, 143), (4098, 129, 3), (20000, 64, 2),
                                        (20000, 70, 5000), (9000, 128, 4500), (9000, 250, 30), (30000, 5, 3), (30000, 7, 10000), (6007, 16, 6007)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_narrow_rows(T, D, groups, dtype):
    # several rows to a wavefront: parts of a chunk, groups of the gate shorter and longer than a part
    q8t = require_gpu()
    x = _inputs(T, D, dtype, True, groups)
    _check_fwd(q8t, x, 0.2)
    _check_bwd(q8t, x, 0.2)


@pytest.mark.parametrize("D", [9, 15, 513, 519, 1025, 2047, 5119, 8191])
@pytest.mark.parametrize("post,gated,p", [(True, 1, 0.1), (True, 0, 0.0), (False, 2, 0.1), (False, 1, 0.0), (True, 2, 0.0)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_that_end_inside_eight(D, post, gated, p, dtype):
    q8t = require_gpu()
    _check_bwd(q8t, _inputs(21, D, dtype, post, {0: 0, 1: 1, 2: 21}[gated]), p)


def test_parts_left_out():
    q8t = require_gpu()
    import torch
    x = _inputs(40, 300, "float32", True, 1)
    _check_bwd(q8t, x, 0.0, parts=("dy",))
    _check_bwd(q8t, x, 0.1, parts=("dres_out",))
    # the norm in front alone
    y = q8t.residual_norm_fwd(x["res"], None, w_pre=x["w_pre"])
    assert y[0] is None and y[3] is None
    r, w = plain.host(x["res"]), plain.host(x["w_pre"])
    s2 = 1 / np.sqrt((r * r).mean(axis=1) + 1e-6)
    plain.within(y[1], r * s2[:, None] * w, 64 * U * np.abs(r * s2[:, None] * w), "y")
    got = q8t.residual_norm_bwd(x["dy"], None, x["res"], None, y[2], w_pre=x["w_pre"])
    ins = (plain.host(x["dy"]), None, r, None, None, plain.host(y[2])[1], None, None, w, 1.0, 1.0, 1.0)
    want, size = plain.norm_bwd(*ins), plain.norm_bwd(*ins, size=True)
    plain.within(got[0], want[0], 128 * U * size[0], "dres")
    plain.within(got[4], want[4], 168 * U * size[4], "dw_pre")
    assert got[1] is None and got[2] is None and got[3] is None
    # no norm in front
    out = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"])
    assert out[1] is None and torch.equal(out[0], q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], w_pre=x["w_pre"])[0])
    assert q8t.residual_norm_fwd(x["res"], x["h"], w_pre=x["w_pre"], quantized=True, want_y=False)[1] is None


def test_gradients_against_differences():
    # central differences of the plain forward pass in 64 bits along random directions
    q8t = require_gpu()
    x = _inputs(24, 200, "float32", True, 4)
    got = _check_bwd(q8t, x, 0.2)
    H = {k: plain.host(v) for k, v in x.items()}
    keep = plain.kept(24 * 200, 0.2, 55).reshape(24, 200)

    def loss(v):
        r, y, _, _ = plain.norm_fwd(v["res"], v["h"], v["w_post"], v["gate"], v["w_pre"], 1e-6, 0.9, 0.6, keep)
        return (y * H["dy"]).sum() + (r * H["dres_out"]).sum()

    g = np.random.default_rng(0)
    for name, grad in zip(("res", "h", "gate", "w_post", "w_pre"), got):
        d = g.standard_normal(H[name].shape)
        e = 1e-5
        diff = (loss({**H, name: H[name] + e * d}) - loss({**H, name: H[name] - e * d})) / (2 * e)
        # the kernel's share: some 300 roundings of every gradient entry; the differences': 1e-10 of the step
        assert abs(diff - (plain.host(grad) * d).sum()) <= 512 * U * np.sqrt(d.size) * np.sqrt(((plain.host(grad) * d) ** 2).sum()) + 1e-5


def test_rows_of_zeros_and_special_values():
    q8t = require_gpu()
    import torch
    x = _inputs(8, 260, "float32", True, 0)
    x["res"][2] = 0
    x["h"][2] = 0
    x["h"][4, 5] = float("nan")
    x["res"][6, 259] = float("inf")
    r, y, stats, q, s = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], w_pre=x["w_pre"], quantized=True)
    assert not bool(r[2].any()) and not bool(y[2].any()) and not bool(q[2].float().any())
    assert bool(y[4].isnan().all()) and int(r[6].isfinite().sum()) == 259
    others = [0, 1, 2, 3, 5, 7]
    assert bool(y[others].isfinite().all()) and bool(q[others].float().isfinite().all())


def test_dropped_positions_take_nothing():
    q8t = require_gpu()
    import torch
    x = _inputs(5, 123, "float32", False, 0)
    keep = torch.from_numpy(plain.kept(5 * 123, 0.5, 3).reshape(5, 123) != 0).to("cuda:0")
    want = q8t.residual_norm_fwd(x["res"], x["h"], w_pre=x["w_pre"], p=0.5, seed=3)
    x["h"][~keep] = float("nan")
    got = q8t.residual_norm_fwd(x["res"], x["h"], w_pre=x["w_pre"], p=0.5, seed=3)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    everything = q8t.residual_norm_fwd(x["res"], x["h"], w_pre=x["w_pre"], p=1.0, seed=3)
    assert torch.equal(everything[0], x["res"])


def test_no_rows():
    q8t = require_gpu()
    import torch
    e, w = torch.zeros(0, 24, device="cuda:0"), torch.ones(24, device="cuda:0")
    out = q8t.residual_norm_fwd(e, e, w_post=w, w_pre=w, quantized=True)
    assert out[0].shape == (0, 24) and out[3].shape == (0, 128)
    back = q8t.residual_norm_bwd(e, None, e, e, out[2], w_post=w, gate=torch.ones(3, 24, device="cuda:0"), w_pre=w)
    assert all(t.shape == s and not bool(t.any()) for t, s in zip(back[2:], ((3, 24), (24,), (24,))))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_other_ranks_and_offsets(dtype):
    q8t = require_gpu()
    import torch
    x = _inputs(12, 333, dtype, True, 1)
    want = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"])
    buf = torch.zeros(12 * 333 + 1, dtype=x["res"].dtype, device="cuda:0")
    view = buf[1:].view(3, 4, 333)
    view.copy_(x["res"].view(3, 4, 333))
    got = q8t.residual_norm_fwd(view, x["h"].view(3, 4, 333), w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"])
    assert got[0].shape == (3, 4, 333) and torch.equal(got[0].view(12, 333), want[0]) and torch.equal(got[1].view(12, 333), want[1])


def test_in_place_through_the_c_calls():
    q8t = require_gpu()
    import torch
    L = q8t.binding._lib
    x = _inputs(9, 1000, "bfloat16", True, 0)
    want = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], w_pre=x["w_pre"])
    res, y, stats = x["res"].clone(), torch.empty_like(x["res"]), torch.empty(2, 9, device="cuda:0")
    st = torch.cuda.current_stream().cuda_stream
    p = lambda t: t.data_ptr()   # noqa: E731
    assert L.q8t_residual_norm_fwd(p(res), p(x["h"]), p(x["w_post"]), None, 0, p(x["w_pre"]), 1, 9, 1000, 1e-6, 1.0, 1.0, 0.0, 0, None, p(res), p(y),
                                   p(stats), None, None, st) == 0
    assert torch.equal(res, want[0]) and torch.equal(y, want[1])
    grads = q8t.residual_norm_bwd(x["dy"], x["dres_out"], want[0], x["h"], want[2], w_post=x["w_post"], w_pre=x["w_pre"])
    for into in ("dy", "dres_out"):
        t = {k: x[k].clone() for k in ("dy", "dres_out")}
        dh, wp, wq = torch.empty_like(x["h"]), torch.empty(1000, device="cuda:0"), torch.empty(1000, device="cuda:0")
        ws = torch.empty(L.q8t_residual_norm_bwd_workspace_size(9, 1000, 0), dtype=torch.uint8, device="cuda:0")
        assert L.q8t_residual_norm_bwd(p(t["dy"]), p(t["dres_out"]), p(want[0]), p(x["h"]), p(want[2]), p(x["w_post"]), None, 0, p(x["w_pre"]), 1, 9,
                                       1000, 1.0, 1.0, 0.0, 0, None, p(t[into]), p(dh), None, p(wp), p(wq), p(ws), st) == 0
        assert torch.equal(t[into], grads[0]) and torch.equal(dh, grads[1]) and torch.equal(wp, grads[3]) and torch.equal(wq, grads[4])


@pytest.mark.parametrize("D", [9, 100, 515, 4100, 5120, 8200, 12290, 16384])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradient_over_an_input_through_the_c_call(D, dtype):
    q8t = require_gpu()
    import torch
    L = q8t.binding._lib
    T, dt = 40, getattr(torch, dtype)
    x = _inputs(T, D, dtype, True, 1)
    fwd = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], p=0.1, seed=3)
    H, s = {k: plain.host(v) for k, v in x.items()}, plain.host(fwd[2])
    keep = plain.kept(T * D, 0.1, 3).reshape(T, D)
    ins = (H["dy"], H["dres_out"], plain.host(fwd[0]), H["h"], s[0], s[1], H["w_post"], H["gate"], H["w_pre"], 1.0, 1.0, keep)
    want, size = plain.norm_bwd(*ins), plain.norm_bwd(*ins, size=True)
    p = lambda t: t.data_ptr()   # noqa: E731
    for into in ("dy", "dres_out"):
        t = {k: x[k].clone() for k in ("dy", "dres_out")}
        dh, dg = torch.empty_like(x["h"]), torch.empty_like(x["gate"])
        wp, wq = torch.empty(D, device="cuda:0"), torch.empty(D, device="cuda:0")
        ws = torch.empty(L.q8t_residual_norm_bwd_workspace_size(T, D, 1), dtype=torch.uint8, device="cuda:0")
        assert L.q8t_residual_norm_bwd(p(t["dy"]), p(t["dres_out"]), p(fwd[0]), p(x["h"]), p(fwd[2]), p(x["w_post"]), p(x["gate"]), 1, p(x["w_pre"]),
                                       int(dt == torch.bfloat16), T, D, 1.0, 1.0, 0.1, 3, None, p(t[into]), p(dh), p(dg), p(wp), p(wq), p(ws),
                                       torch.cuda.current_stream().cuda_stream) == 0
        for name, g, w, z in zip(("dres", "dh", "dgate", "dw_post", "dw_pre"), (t[into], dh, dg, wp, wq), want, size):
            rows = T if name[:2] == "dw" or name == "dgate" else 0           # as in _check_bwd
            plain.within(g, w, plain.HALF[g.dtype] * np.abs(w) + (128 + rows) * U * z, name)


def test_beyond_32_bits():
    q8t = require_gpu()
    import torch
    T, D = 262200, 8200
    res = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda:0")
    x = _inputs(60, D, "bfloat16", True, 1)
    res[-60:] = x["res"]
    h = torch.zeros_like(res)
    h[-60:] = x["h"]
    got = q8t.residual_norm_fwd(res, h, w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], quantized=True)
    want = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], quantized=True)
    assert torch.equal(got[0][-60:], want[0]) and torch.equal(got[1][-60:], want[1])
    assert torch.equal(got[3][-60:].view(torch.uint8), want[3].view(torch.uint8))
    dy = torch.zeros_like(res)
    dy[-60:] = x["dy"]
    back = q8t.residual_norm_bwd(dy, None, got[0], h, got[2], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"])
    small = q8t.residual_norm_bwd(x["dy"], None, want[0], x["h"], want[2], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"])
    assert torch.equal(back[0][-60:], small[0]) and torch.equal(back[1][-60:], small[1]) and not bool(back[1][:-60].any())


def test_captured_and_on_two_streams():
    q8t = require_gpu()
    import torch
    xs = [_inputs(300, 520, "bfloat16", True, 3, seed=k) for k in range(2)]
    step = torch.zeros(1, dtype=torch.int64, device="cuda:0")

    def call(x, seed=5, step=None):
        f = q8t.residual_norm_fwd(x["res"], x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], p=0.1, seed=seed, step=step)
        return f[:3] + q8t.residual_norm_bwd(x["dy"], x["dres_out"], f[0], x["h"], f[2], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"], p=0.1,
                                             seed=seed, step=step)

    want = [call(x) for x in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for _ in range(5):
        for k, (s, x) in enumerate(zip(streams, xs)):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append((k, call(x)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for k, r in got for a, b in zip(r, want[k]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(xs[0], step=step)
        step.add_(1)
    step.zero_()
    for k in range(3):
        graph.replay()
        eager = call(xs[0], seed=5 + k)
        call(xs[1])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager))


def test_refusals():
    q8t = require_gpu()
    import torch
    x = _inputs(6, 64, "float32", True, 2)
    f = lambda **k: q8t.residual_norm_fwd(x["res"], **{**dict(h=x["h"], w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"]), **k})   # noqa: E731
    for k in (dict(h=x["h"][:3]), dict(h=x["h"].bfloat16()), dict(w_post=x["w_post"][:32]), dict(w_post=x["w_post"].bfloat16()), dict(gate=x["gate"][0]),
              dict(gate=x["gate"][:, :32].contiguous()), dict(gate=torch.ones(4, 64, device="cuda:0")), dict(w_pre=x["w_pre"].double()), dict(h=None),
              dict(p=-1.0), dict(p=2.0), dict(h=None, w_post=None, gate=None, p=0.5), dict(h=None, w_post=None, gate=None, res_scale=2.0),
              dict(h=None, w_post=None, gate=None, w_pre=None), dict(w_pre=None, quantized=True), dict(h=x["h"].t().contiguous().t()), dict(w_pre=x["w_pre"].cpu())):
        with pytest.raises((ValueError, q8t.Q8TError)):
            f(**k)
    with pytest.raises(q8t.Q8TError, match="SHAPE"):
        wide = torch.zeros(1, 16385, device="cuda:0")
        q8t.residual_norm_fwd(wide, wide)
    out = f()
    b = lambda *a, **k: q8t.residual_norm_bwd(*a, **{**dict(w_post=x["w_post"], gate=x["gate"], w_pre=x["w_pre"]), **k})   # noqa: E731
    for a, k in (((None, None, out[0], x["h"], out[2]), {}), ((x["dy"], None, out[0], None, out[2]), {}), ((x["dy"], None, out[0], x["h"], None), {}),
                 ((x["dy"], None, out[0], x["h"], out[2][:, :3].contiguous()), {}), ((x["dy"], None, out[0], x["h"], out[2]), dict(w_pre=None)),
                 ((x["dy"].bfloat16(), None, out[0], x["h"], out[2]), {}),
                 ((x["dy"], None, out[0], x["h"], out[2]), dict(ws=torch.empty(16, device="cuda:0")))):
        with pytest.raises((ValueError, q8t.Q8TError)):
            b(*a, **k)
