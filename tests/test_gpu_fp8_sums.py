"""What a product of 8-bit floating point codes keeps of its sums: small terms beside large ones that cancel."""
import numpy as np
import pytest

import lm_plain as plain
from fp8_forms import FORMS
from gpu_util import require_gpu

pytestmark = pytest.mark.gpu

# products of few rows, which read their operands straight to registers
FEW = [(1, 4093, 4100), (1, 100, 300), (16, 48, 640), (64, 70, 130), (13, 300, 1030), (29, 4090, 4000), (61, 515, 2000), (61, 4090, 4000)]


def _device(q, s, fmt):
    import torch
    code = torch.float8_e4m3fn if fmt == "e4m3" else torch.float8_e5m2
    return torch.from_numpy(q).to(torch.float32).to(code).to("cuda:0"), torch.from_numpy(s).to("cuda:0").view(torch.float8_e8m0fnu)


def _cancelling(M, N, K, fa, fb):
    """Codes and scales on the device, and the exact product: in each block 1 and -1, and 2^-16 or -2^-16 for every other entry.  All sums are
    whole numbers of 2^-16 below 2^7, exact in fp32 in any order."""
    g = np.random.default_rng(M + N + K)
    nb = K // 128
    Kp = -(-K // 128) * 128
    a, b = np.zeros((M, Kp)), np.zeros((N, Kp))
    a[:, :K] = g.choice([-1.0, 1.0], (M, K)) * 2.0 ** -8
    b[:, :K] = g.choice([-1.0, 1.0], (N, K)) * 2.0 ** -8
    sign = g.choice([-1.0, 1.0], (M, nb))
    for k in range(nb):
        at = 128 * k + g.choice(128, 2, replace=False)
        a[:, at] = sign[:, k, None] * np.array([1.0, -1.0])
        b[:, at] = 1.0
    ones = [np.full((R, -(-Kp // 512) * 4), 127, np.uint8) for R in (M, N)]
    want = (a.astype(np.float32) * np.float32(2 ** 8)) @ (b.astype(np.float32) * np.float32(2 ** 8)).T * np.float32(2.0 ** -16)
    assert np.abs(want).max() < 128
    return _device(a, ones[0], fa) + _device(b, ones[1], fb), want


@pytest.mark.parametrize("M,N,K", FEW)
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e4m3", "e5m2"), ("e5m2", "e4m3")])
def test_few_rows_to_bf16_are_summed_in_fp32(M, N, K, fa, fb):
    q8t = require_gpu()
    import torch
    ops, want = _cancelling(M, N, K, fa, fb)
    assert torch.equal(q8t.fp8_gemm(*ops).cpu(), torch.from_numpy(want).bfloat16())


@pytest.mark.parametrize("M,N,K", FEW + [(20, 30, 256)])
def test_few_rows_to_bf16_at_the_ends_of_the_scales(M, N, K):
    # what codes and scales stand for: below bf16's last place, 2^-133, or above its largest number, next to rows of ordinary scales
    q8t = require_gpu()
    K = K // 128 * 128
    for code, ea, eb in ((2.0 ** -9, 0, 254), (1.0, 0, 254), (448.0, 247, 7), (448.0, 254, 0), (2.0 ** -9, 3, 251), (416.0, 240, 14)):
        a, b = np.full((M, K), code), np.full((N, K), 1.0)
        sa, sb = np.full((M, -(-K // 512) * 4), 127, np.uint8), np.full((N, -(-K // 512) * 4), 127, np.uint8)
        sa[M // 2:, :K // 128] = ea
        sb[N // 2:, :K // 128] = eb
        want = np.full((M, N), code * K)
        scale = np.exp2(sa[:, :1].astype(np.float64) - 127) * np.exp2(sb[:, :1].astype(np.float64).T - 127)
        want = want * scale
        got = plain.host(q8t.fp8_gemm(*(_device(a, sa, "e4m3") + _device(b, sb, "e5m2"))))
        normal = (want >= 2.0 ** -126) & (want < 2.0 ** 128)
        assert normal[M // 2:, N // 2:].all()
        # whole multiples of one product in fp32: below 2^24 of them exact; one rounding to bf16
        off = 2.0 ** -8 * want
        assert (np.abs(got - want)[normal] <= off[normal]).all(), (code, ea, eb)


@pytest.mark.parametrize("M,N,K", FEW)
@pytest.mark.parametrize("scale", [0, 3, 250, 255])
def test_scales_at_the_ends_leave_other_rows_alone(M, N, K, scale):
    # ordinary rows beside a row whose scales are at an end, or stand for NaN, in some blocks: the same bits as without it
    q8t = require_gpu()
    import torch
    g = np.random.default_rng(K)
    (a, sa, _, _), (b, sb, _, _) = (q8t.fp8_quantize(torch.from_numpy(g.standard_normal((R, K), np.float32)).to("cuda:0"), f) for R, f in ((M, "e4m3"), (N, "e5m2")))
    want = q8t.fp8_gemm(a, sa, b, sb)
    rows, cols = torch.arange(M) % 5 != 2, torch.arange(N) % 7 != 3
    sa.view(torch.uint8)[~rows, 1:8:2] = scale
    sb.view(torch.uint8)[~cols, 2:7] = scale
    got = q8t.fp8_gemm(a, sa, b, sb)
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])
    if scale == 255:
        assert bool(got[~rows].isnan().all()) and (K <= 256 or bool(got[:, ~cols].isnan().all()))    # block 2 on: behind the end of 130


# fp32 results: operands straight to registers, tiles of 64 x 64 in one slice and in several, and larger ones
WIDE = [(1, 4093, 4100), (61, 4090, 4000), (250, 500, 1500), (70, 300, 8192), (500, 4090, 4000), (2000, 2100, 1500), (4090, 8200, 2000)]


@pytest.mark.parametrize("M,N,K", WIDE)
def test_fp32_results_at_the_ends_of_the_range_of_codes(M, N, K):
    # 2^-133 and the largest numbers below 2^128 on one side, brought back by the other side's scale: whole multiples of one product
    q8t = require_gpu()
    import torch
    K = K // 128 * 128
    for fa, code, ea, eb in (("e4m3", 2.0 ** -9, 3, 240), ("e4m3", 448.0, 246, 9), ("e5m2", 2.0 ** -16, 10, 240), ("e5m2", 57344.0, 239, 9)):
        a, b = np.full((M, K), code), np.full((N, K), 1.0)
        sa, sb = np.full((M, -(-K // 512) * 4), ea, np.uint8), np.full((N, -(-K // 512) * 4), eb, np.uint8)
        got = q8t.fp8_gemm(*(_device(a, sa, fa) + _device(b, sb, "e4m3")), dtype=torch.float32)
        assert bool((got == code * K * 2.0 ** (ea + eb - 254)).all()), (fa, code)


@pytest.mark.parametrize("M,N,K", [f[:3] for f in FORMS])
@pytest.mark.parametrize("fa,fb", [("e4m3", "e4m3"), ("e4m3", "e5m2")])
def test_fp32_results_keep_small_terms(M, N, K, fa, fb):
    # the 8-bit matrix instruction, which adds in groups of eight, loses most of these terms of 2^-16
    q8t = require_gpu()
    import torch
    ops, want = _cancelling(M, N, K, fa, fb)
    assert torch.equal(q8t.fp8_gemm(*ops, dtype=torch.float32).cpu(), torch.from_numpy(want))


@pytest.mark.parametrize("M,N,K", [f[:3] for f in FORMS])
def test_fp32_results_of_ordinary_values(M, N, K):
    # Error in the 2-norm.  An addition to a partial sum of n terms of variance 1 is off by at most 2^-24 sqrt(n) of its size, and the errors
    # are as good as independent: after K of them at most 2^-24 sqrt(K^2 / 2) beside a result of sqrt(K), 2^-24 sqrt(K / 2): 1.5e-6 at
    # 1300, 5.4e-6 at 16500.  The 8-bit matrix instruction is 0.8e-5 to 1.5e-5 off.
    q8t = require_gpu()
    import torch
    g = np.random.default_rng(K)
    x, y = (torch.from_numpy(g.standard_normal((R, K), np.float32)).to("cuda:0") for R in (M, N))
    (a, sa, _, _), (b, sb, _, _) = q8t.fp8_quantize(x), q8t.fp8_quantize(y, "e5m2")
    A, B = (torch.from_numpy(plain.values(plain.host(q), s.view(torch.uint8).cpu().numpy())) for q, s in ((a, sa), (b, sb)))
    want = A @ B.T
    got = q8t.fp8_gemm(a, sa, b, sb, dtype=torch.float32).cpu().double()
    assert float((got - want).norm() / want.norm()) <= 2.0 ** -24 * (K / 2) ** 0.5
