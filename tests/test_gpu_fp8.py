"""8-bit floating point codes with a scale a block of 128, and their product: against the plain form in 64 bits (lm_plain.py)."""
import numpy as np
import pytest

import lm_plain as plain
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (1, 127), (1, 4096), (3, 129), (17, 128), (128, 128), (127, 131), (129, 260), (200, 515), (300, 1030), (513, 127)]


def _x(R, C, seed, dtype="float32"):
    """values over many octaves, with a large column, an empty block and one single entry in a block"""
    import torch
    g = np.random.default_rng(seed)
    x = g.standard_normal((R, C)) * np.exp(2 * g.standard_normal((R, C)))
    x[:, C // 2] *= 300
    x[R // 2, :128] = 0
    x[R // 2, min(5, C - 1)] = -3e-5
    x[0, :min(C, 128)] = 0
    return torch.from_numpy(x.astype(np.float32)).to(getattr(torch, dtype)).to("cuda:0")


def _check(x, got, fmt, square, r):
    import torch
    hx = plain.host(x)
    rr = None if r is None else r.reshape(hx.shape)
    rows = 128 if square else 1
    pairs = [(got[0], got[1], plain.quantize(hx, fmt, rows, rr))]
    if got[2] is not None:
        pairs.append((got[2], got[3], plain.quantize(hx.T, fmt, rows, None if rr is None else rr.T)))
    for q, s, (wq, ws) in pairs:
        assert np.array_equal(s.view(torch.uint8).cpu().numpy(), ws)
        assert np.array_equal(plain.host(q), wq, equal_nan=True)
        assert np.array_equal(np.signbit(plain.host(q))[wq == wq], np.signbit(wq)[wq == wq])


@pytest.mark.parametrize("R,C", SHAPES)
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("stochastic", [False, True])
def test_codes(R, C, dtype, fmt, stochastic):
    q8t = require_gpu()
    import torch
    x = _x(R, C, R * 7 + C, dtype)
    seed = 0x9876543210ABCDEF
    step = torch.tensor([3], device="cuda:0")
    r = plain.draws(R * C, seed + 3) if stochastic else None
    for square in (False, True):
        for both in (False, True):
            got = q8t.fp8_quantize(x, fmt, square=square, stochastic=stochastic, seed=seed, step=step, transposed=both)
            assert (got[2] is not None) == both
            _check(x, got, fmt, square, r)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("stochastic", [False, True])
def test_special_values(fmt, stochastic):
    q8t = require_gpu()
    import torch
    x = _x(140, 300, 5)
    x[1, 3], x[1, 140], x[2, 7], x[130, 299] = float("inf"), -float("inf"), float("nan"), float("inf")
    x[5, :128] = float("nan")                                # nothing finite in a block
    x[7, :128] = 1e-42                                       # denormal values
    x[8, :128] = 3.4e38
    x[9, :128] = 448.0 * 2.0 ** -20
    x[10, 0:128] = torch.nextafter(torch.tensor(448.0), torch.tensor(1000.0)).item()
    x[11, :128] = torch.arange(128, device="cuda:0") / 64.0 + 1.0 / 32    # ties of the coarser steps
    r = plain.draws(140 * 300, 1) if stochastic else None
    _check(x, q8t.fp8_quantize(x, fmt, stochastic=stochastic, seed=1, transposed=True), fmt, False, r)
    _check(x, q8t.fp8_quantize(x, fmt, stochastic=stochastic, seed=1), fmt, False, r)
    _check(x, q8t.fp8_quantize(x, fmt, stochastic=stochastic, seed=1, square=True, transposed=True), fmt, True, r)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scales_at_the_lower_end(fmt, dtype):
    # blocks of a scale under the smallest normal number's, over rows, over columns, and next to others; denormal values among them
    q8t = require_gpu()
    import torch
    g = np.random.default_rng(8)
    x = g.standard_normal((260, 300)) * np.exp2(g.integers(-149, -90, (260, 300)))
    x[:128, 128:] *= 2.0 ** 80
    x[:, 7] *= 2.0 ** 30
    x = torch.from_numpy(x).to(getattr(torch, dtype)).to("cuda:0")
    r = plain.draws(260 * 300, 1)
    for square in (False, True):
        for both in (False, True):
            _check(x, q8t.fp8_quantize(x, fmt, square=square, transposed=both), fmt, square, None)
            _check(x, q8t.fp8_quantize(x, fmt, square=square, stochastic=True, seed=1, transposed=both), fmt, square, r)


@pytest.mark.parametrize("dtype,off", [("float32", 1), ("bfloat16", 1), ("bfloat16", 3)])
def test_quantize_view_at_an_offset(dtype, off):
    q8t = require_gpu()
    R, C = 131, 256
    flat = _x(1, R * C + off, 9, dtype).view(-1)
    x = flat[off:].view(R, C)
    for both in (False, True):
        _check(x, q8t.fp8_quantize(x, "e4m3", transposed=both), "e4m3", False, None)


def test_quantize_writes_its_rows_alone():
    q8t = require_gpu()
    import torch
    R, C = 130, 200
    x = _x(R, C, 2)
    bufs = [torch.full((n + 3, w), 0x55, dtype=torch.uint8, device="cuda:0") for n, w in ((R, 256), (R, 4), (C, 256), (C, 4))]
    types = [torch.float8_e4m3fn, torch.float8_e8m0fnu] * 2
    outs = [b[:n].view(t) for b, n, t in zip(bufs, (R, R, C, C), types)]
    for both in (False, True):
        q8t.fp8_quantize(x, "e4m3", transposed=both, q_out=outs[0], s_out=outs[1], qt_out=outs[2], st_out=outs[3])
        torch.cuda.synchronize()
        for b, n in zip(bufs, (R, R, C, C)):
            assert bool((b[n:] == 0x55).all())
    _check(x, outs, "e4m3", False, None)


def test_quantize_empty():
    q8t = require_gpu()
    import torch
    for R, C in ((0, 5), (5, 0), (0, 0)):
        q, s, qt, st = q8t.fp8_quantize(torch.zeros(R, C, device="cuda:0"), transposed=True)
        assert q.shape[0] == R and qt.shape[0] == C


def test_quantize_beyond_32_bits():
    q8t = require_gpu()
    import torch
    R, C = 65540, 32784
    x = torch.zeros(R, C, dtype=torch.bfloat16, device="cuda:0")
    tail = _x(132, C, 4, "bfloat16")
    x[-132:] = tail
    q, s, qt, st = q8t.fp8_quantize(x, "e4m3", transposed=True)
    only = q8t.fp8_quantize(x, "e4m3")
    want = q8t.fp8_quantize(tail, "e4m3")
    assert torch.equal(q[-132:].view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(s[-132:].view(torch.uint8), want[1].view(torch.uint8))
    assert torch.equal(only[0][-132:].view(torch.uint8), want[0].view(torch.uint8))
    last = q8t.fp8_quantize(x[65408:].contiguous(), "e4m3", transposed=True)     # the columns' last two blocks: 65408 = 511 * 128
    assert torch.equal(qt[:, 65408:].contiguous().view(torch.uint8), last[2].view(torch.uint8))
    assert torch.equal(st[:, 511:513].contiguous().view(torch.uint8), last[3][:, :2].contiguous().view(torch.uint8))


# ---------------------------------------------------------------------------------------- products
PRODUCTS = [(1, 1, 1), (1, 16, 128), (1, 4096, 512), (1, 1000, 4100), (2, 17, 129), (16, 48, 640), (17, 33, 1000), (5, 300, 2049), (33, 1, 700),
            (64, 64, 128), (65, 127, 384), (128, 128, 512), (200, 1000, 515), (129, 257, 1025), (256, 256, 256), (255, 513, 130), (300, 520, 4097),
            (513, 1030, 260), (640, 768, 1536), (1, 20, 16384), (24, 40, 16500), (128, 256, 8200), (1000, 1100, 700), (2000, 2100, 390), (4200, 4100, 140), (70, 300, 8192)]


def _operand(R, K, fmt, seed, whole=False):
    """codes and scales on the device, and what they stand for.  whole: small whole numbers times 1, 2 or 4, so that every sum of up to
    2^24 / 16^2 / 16 products is exact in fp32 in any order"""
    import torch
    g = np.random.default_rng(seed)
    if whole:
        Kp, nb = -(-K // 128) * 128, -(-K // 128)
        q = np.zeros((R, Kp))
        q[:, :K] = g.integers(-3, 4, (R, K))
        s = np.full((R, -(-nb // 4) * 4), 127, np.uint8)
        s[:, :nb] += g.integers(0, 3, (R, nb)).astype(np.uint8)
    else:
        x = g.standard_normal((R, K)) * np.exp(g.standard_normal((R, 1)))
        q, s = plain.quantize(x, fmt)
    code = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    return (torch.from_numpy(q).to(torch.float32).to(code).to("cuda:0"), torch.from_numpy(s).to("cuda:0").view(torch.float8_e8m0fnu),
            plain.values(q, s))


@pytest.mark.parametrize("M,N,K", PRODUCTS)
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e5m2", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e5m2")])
def test_product_exact_sums(M, N, K, fa, fb):
    q8t = require_gpu()
    import torch
    a, sa, va = _operand(M, K, fa, 1, whole=True)
    b, sb, vb = _operand(N, K, fb, 2, whole=True)
    want = va @ vb.T
    assert (np.abs(va) @ np.abs(vb).T).max() < 2 ** 24
    got = q8t.fp8_gemm(a, sa, b, sb, dtype=torch.float32)
    assert np.array_equal(plain.host(got), want)
    got = q8t.fp8_gemm(a, sa, b, sb)
    assert got.dtype == torch.bfloat16 and np.array_equal(plain.host(got), plain.host(torch.from_numpy(want).to(torch.float32).bfloat16()))


@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product_of_ordinary_values(M, N, K):
    # fp32: a sum of K products in any order: K - 1 additions, each off by at most one unit in the last place of a partial sum,
    # which is at most the sum of magnitudes.  bf16: the 8-bit matrix instruction, which adds products in groups of eight and loses
    # of seven of them up to 2^-13 of the largest each, so less than 2^-10 of the sum of magnitudes, and one rounding of the result
    q8t = require_gpu()
    import torch
    a, sa, va = _operand(M, K, "e4m3", 3)
    b, sb, vb = _operand(N, K, "e5m2", 4)
    want, size = va @ vb.T, np.abs(va) @ np.abs(vb).T
    off = K * 2.0 ** -23 * size
    plain.within(q8t.fp8_gemm(a, sa, b, sb, dtype=torch.float32), want, off, (M, N, K))
    off = off + 2.0 ** -10 * size
    plain.within(q8t.fp8_gemm(a, sa, b, sb), want, off + 2.0 ** -8 * (np.abs(want) + off), (M, N, K))


@pytest.mark.parametrize("M,N,K", [(4101, 4093, 1100), (1024, 4090, 1500), (500, 4100, 3000), (1003, 3000, 2000), (8192, 260, 1000), (6000, 6100, 250),
                                   (100, 9000, 5000), (1, 30000, 2000), (16, 20000, 1030)])
def test_large_products(M, N, K):
    # whole numbers whose sums stay below 2^24: the same in fp32 in any order
    q8t = require_gpu()
    import torch
    a, sa, va = _operand(M, K, "e4m3", 5, whole=True)
    b, sb, vb = _operand(N, K, "e5m2", 6, whole=True)
    assert 144 * K < 2 ** 24
    want = torch.from_numpy(va.astype(np.float32) @ vb.astype(np.float32).T)
    assert torch.equal(q8t.fp8_gemm(a, sa, b, sb, torch.float32).cpu(), want)
    assert torch.equal(q8t.fp8_gemm(a, sa, b, sb).cpu(), want.bfloat16())


@pytest.mark.parametrize("M,N,K", [(1, 100, 300), (40, 70, 260), (300, 300, 700), (520, 530, 256)])
def test_a_nan_stays_in_its_row(M, N, K):
    q8t = require_gpu()
    import torch
    a, sa, va = _operand(M, K, "e4m3", 1, whole=True)
    b, sb, vb = _operand(N, K, "e5m2", 2, whole=True)
    m, n = M - 1, N // 2
    a[m, K - 1] = float("nan")
    b[n, 0] = float("inf")
    got = plain.host(q8t.fp8_gemm(a, sa, b, sb, dtype=torch.float32))
    clean = np.ones((M, N), bool)
    clean[m, :] = clean[:, n] = False
    assert np.isnan(got[m]).all() and not np.isfinite(got[:, n]).any()
    assert np.array_equal(got[clean], (va @ vb.T)[clean])


@pytest.mark.parametrize("M,N,K", [(1, 100, 300), (40, 70, 260), (300, 300, 700), (520, 530, 256), (600, 3000, 256)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_a_scale_that_is_none_stays_in_its_row(M, N, K, dtype):
    # scale 255 stands for NaN
    q8t = require_gpu()
    import torch
    a, sa, va = _operand(M, K, "e4m3", 1, whole=True)
    b, sb, vb = _operand(N, K, "e5m2", 2, whole=True)
    m, n = M - 1, N // 2
    sa.view(torch.uint8)[m, 1] = 255
    sb.view(torch.uint8)[n, 0] = 255
    got = q8t.fp8_gemm(a, sa, b, sb, dtype=getattr(torch, dtype))
    clean = np.ones((M, N), bool)
    clean[m, :] = clean[:, n] = False
    assert np.isnan(plain.host(got)[~clean]).all()
    want = torch.from_numpy(va @ vb.T).to(torch.float32).to(got.dtype)
    assert np.array_equal(plain.host(got)[clean], plain.host(want)[clean])


@pytest.mark.parametrize("M,N,K", [(1, 130, 300), (37, 100, 200), (260, 300, 300), (513, 514, 1280)])
def test_product_writes_its_rows_alone(M, N, K):
    q8t = require_gpu()
    import torch
    a, sa, va = _operand(M, K, "e4m3", 1, whole=True)
    b, sb, vb = _operand(N, K, "e4m3", 2, whole=True)
    for dtype in (torch.float32, torch.bfloat16):
        buf = torch.full((N + 7 + M * N,), -7.0, dtype=dtype, device="cuda:0")
        out = buf[3:3 + M * N].view(M, N)       # at an odd offset
        q8t.fp8_gemm(a, sa, b, sb, dtype=dtype, out=out)
        assert bool((buf[:3] == -7).all()) and bool((buf[3 + M * N:] == -7).all())
        assert np.array_equal(plain.host(out), plain.host(torch.from_numpy(va @ vb.T).to(torch.float32).to(dtype)))


def test_smallest_and_largest_scales():
    q8t = require_gpu()
    import torch
    K = 256
    for ea, eb in ((0, 254), (254, 0), (7, 247), (120, 134)):   # 2^(ea - 127) 2^(eb - 127) between 1 and 2^4
        a = torch.full((20, K), 1.5).to(torch.float8_e4m3fn).to("cuda:0")
        b = torch.full((30, K), -1.0).to(torch.float8_e5m2).to("cuda:0")
        sa = torch.full((20, 4), ea, dtype=torch.uint8, device="cuda:0").view(torch.float8_e8m0fnu)
        sb = torch.full((30, 4), eb, dtype=torch.uint8, device="cuda:0").view(torch.float8_e8m0fnu)
        got = q8t.fp8_gemm(a, sa, b, sb, dtype=torch.float32)
        assert bool((got == -1.5 * K * 2.0 ** (ea + eb - 254)).all())


def test_product_empty():
    q8t = require_gpu()
    a, sa, _ = _operand(4, 100, "e4m3", 1)
    for x, y in ((0, 4), (4, 0), (0, 0)):
        assert q8t.fp8_gemm(a[:x], sa[:x], a[:y], sa[:y]).shape == (x, y)


def test_product_beyond_32_bits():
    q8t = require_gpu()
    import torch
    M, N, K = 65600, 32800, 128
    a, sa, va = _operand(200, K, "e4m3", 1, whole=True)
    b, sb, vb = _operand(N, K, "e4m3", 2, whole=True)
    big = torch.zeros(M, K, dtype=torch.uint8, device="cuda:0").view(torch.float8_e4m3fn)
    bigs = torch.full((M, 4), 127, dtype=torch.uint8, device="cuda:0").view(torch.float8_e8m0fnu)
    big[-200:], bigs[-200:] = a, sa
    out = q8t.fp8_gemm(big, bigs, b, sb)
    want = q8t.fp8_gemm(a, sa, b, sb)
    assert torch.equal(out[-200:], want) and not bool(out[:-200].any())
    assert np.array_equal(plain.host(want), plain.host(torch.from_numpy(va @ vb.T).to(torch.float32).bfloat16()))


def test_layer_products_follow_from_the_copies():
    # Y = X W, dX = dY W^T, dW = X^T dY with the operands that one quantization of each tensor leaves
    q8t = require_gpu()
    import torch
    M, K, N = 150, 300, 200
    x, w, dy = _x(M, K, 1), _x(K, N, 2), _x(M, N, 3)
    qx, sx, xt, sxt = q8t.fp8_quantize(x, transposed=True)
    qw, sw, wt, swt = q8t.fp8_quantize(w, square=True, transposed=True)
    qg, sg, gt, sgt = q8t.fp8_quantize(dy, "e5m2", stochastic=True, seed=4, transposed=True)
    v = lambda q, s, n: plain.values(plain.host(q), s.view(torch.uint8).cpu().numpy())[:, :n]   # noqa: E731
    W = v(qw, sw, N)
    assert np.array_equal(W, v(wt, swt, K).T)
    for got, A, B in ((q8t.fp8_gemm(qx, sx, wt, swt, torch.float32), v(qx, sx, K), W), (q8t.fp8_gemm(qg, sg, qw, sw, torch.float32), v(qg, sg, N), W.T),
                      (q8t.fp8_gemm(xt, sxt, gt, sgt, torch.float32), v(xt, sxt, M), v(gt, sgt, M).T)):
        plain.within(got, A @ B, A.shape[1] * 2.0 ** -23 * (np.abs(A) @ np.abs(B)), A.shape)


@pytest.mark.parametrize("M,N,K", [(3, 5000, 4096), (200, 1000, 515), (700, 900, 2000)])
def test_streams_and_graph(M, N, K):
    q8t = require_gpu()
    import torch
    ops = [[_operand(M, K, "e4m3", 10 + i), _operand(N, K, "e4m3", 20 + i)] for i in range(2)]
    call = lambda i: q8t.fp8_gemm(ops[i][0][0], ops[i][0][1], ops[i][1][0], ops[i][1][1], torch.float32)   # noqa: E731
    want = [call(0), call(1)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(6):
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append((i, call(i)))
    torch.cuda.synchronize()
    assert all(torch.equal(t, want[i]) for i, t in got)
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call(i)
        graphs.append((g, out))
    for _ in range(3):
        for i, (g, out) in enumerate(graphs):
            out.zero_()
            g.replay()
            eager = call(1 - i)
            torch.cuda.synchronize()
            assert torch.equal(out, want[i]) and torch.equal(eager, want[1 - i])


def test_refusals():
    q8t = require_gpu()
    import torch
    x = torch.zeros(8, 256, device="cuda:0")
    q, s, _, _ = q8t.fp8_quantize(x)
    for call in (lambda: q8t.fp8_quantize(x, "e3m4"), lambda: q8t.fp8_quantize(x.half()), lambda: q8t.fp8_quantize(x[0]),
                 lambda: q8t.fp8_quantize(x.t()), lambda: q8t.fp8_quantize(x, q_out=q[:4]), lambda: q8t.fp8_quantize(x, s_out=q),
                 lambda: q8t.fp8_quantize(x, "e5m2", q_out=q), lambda: q8t.fp8_gemm(q, s, q, s, torch.float16),
                 lambda: q8t.fp8_gemm(q, s, q[:, :128].contiguous(), s), lambda: q8t.fp8_gemm(q, s[:4], q, s),
                 lambda: q8t.fp8_gemm(q.view(torch.uint8), s, q, s), lambda: q8t.fp8_gemm(q, s.view(torch.uint8), q, s),
                 lambda: q8t.fp8_gemm(q, s, q, s, out=torch.zeros(8, 8, device="cuda:0")), lambda: q8t.fp8_gemm(q, s, q.cpu(), s),
                 lambda: q8t.fp8_gemm(q, s, q, s, ws=torch.empty(16, device="cuda:0").t()[:0].cpu()),
                 lambda: q8t.fp8_gemm(q[:, 64:192], s, q, s), lambda: q8t.fp8_gemm(q[:, :0], s[:, :0], q[:, :0], s[:, :0])):
        with pytest.raises((ValueError, q8t.Q8TError)):
            call()
    a, sa, _, _ = q8t.fp8_quantize(torch.zeros(512, 8192, device="cuda:0"))     # summed in slices
    assert q8t.binding._lib.q8t_fp8_gemm_workspace_size(512, 512, 8192) > 1024
    with pytest.raises(ValueError, match="ws"):
        q8t.fp8_gemm(a, sa, a, sa, ws=torch.empty(1024, dtype=torch.uint8, device="cuda:0"))
    flat = torch.zeros(8 * 256 + 8, dtype=torch.uint8, device="cuda:0")
    odd = flat[8:].view(8, 256).view(torch.float8_e4m3fn)        # 8 bytes off a 16-byte address
    for call in (lambda: q8t.fp8_gemm(odd, s, q, s), lambda: q8t.fp8_gemm(q, s, odd, s), lambda: q8t.fp8_quantize(x, q_out=odd)):
        with pytest.raises(q8t.Q8TError, match="SHAPE"):
            call()
