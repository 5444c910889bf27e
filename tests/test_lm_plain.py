"""The plain forms that the GPU tests of the language-model layer compare with, against torch's own conversions and differences (CPU)."""
import numpy as np
import pytest
import torch

import lm_layer
import lm_plain as plain
import oracle


def test_draws_are_those_of_the_oracle():
    for seed in (0, 7, 0x1234567890ABCDEF, 2 ** 64 - 1):
        assert np.array_equal(plain.draws(1003, seed), [oracle.r16(i, seed) for i in range(1003)])


@pytest.mark.parametrize("fmt,dtype", [("e4m3", torch.float8_e4m3fn), ("e5m2", torch.float8_e5m2)])
def test_nearest_codes_are_torchs_conversion_of_the_scaled_values(fmt, dtype):
    g = np.random.default_rng(3)
    x = (g.standard_normal((40, 700)) * np.exp(3 * g.standard_normal((40, 700)))).astype(np.float32).astype(np.float64)
    x[3] = 0
    x[5, :128] = 448.0
    x[6, :128] = np.nextafter(np.float32(448.0), np.float32(500.0))
    q, s = plain.quantize(x, fmt)
    scale = np.exp2(s[:, :6].astype(np.float64) - 127)
    t = np.pad(x, ((0, 0), (0, 68))).reshape(40, 6, 128) / scale[:, :, None]
    assert np.array_equal(q.reshape(40, 6, 128), torch.from_numpy(t).to(torch.float32).to(dtype).double().numpy())
    top = 448.0 if fmt == "e4m3" else 57344.0
    amax = np.abs(t).max(axis=2)
    assert (amax <= top).all() and (amax[amax > 0] > top / 2).all()
    assert (s[3, :6] == 127).all() and (s[:, 6:] == 127).all()


def test_stochastic_codes_are_unbiased():
    x = np.full((1, 128), 1.03)
    x[0, 0] = 448.0
    mean = np.mean([plain.quantize(x, "e4m3", 1, plain.draws(128, seed))[0] for seed in range(400)], axis=0)
    # 50800 draws between neighbours 0.125 apart: the mean is off by at most 5 standard deviations
    assert abs(mean[0, 1:].mean() - 1.03) < 5 * 0.0625 / np.sqrt(400 * 127)


def test_gradients_against_differences():
    g = np.random.default_rng(1)
    T, D, G = 6, 10, 3
    res, h, dy, dro = (g.standard_normal((T, D)) for _ in range(4))
    wp, wq, gate = g.standard_normal(D), g.standard_normal(D), g.standard_normal((G, D))
    keep = (g.random((T, D)) > 0.3) / 0.7
    args = dict(eps=1e-3, rs=0.9, bs=0.7, keep=keep)

    def loss(res, h, gate, wp, wq):
        r, y, _, _ = plain.norm_fwd(res, h, wp, gate, wq, **args)
        return (y * dy).sum() + (r * dro).sum()

    r, _, s1, s2 = plain.norm_fwd(res, h, wp, gate, wq, **args)
    grads = plain.norm_bwd(dy, dro, r, h, s1, s2, wp, gate, wq, 0.9, 0.7, keep)
    for k, t in enumerate((res, h, gate, wp, wq)):
        d = g.standard_normal(t.shape)
        ins = [[v + (sign * 1e-5 * d if i == k else 0) for i, v in enumerate((res, h, gate, wp, wq))] for sign in (1, -1)]
        diff = (loss(*ins[0]) - loss(*ins[1])) / 2e-5
        assert abs(diff - (grads[k] * d).sum()) < 1e-7 * max(1, abs(diff))   # 1e-10 of the step, 1e-11 of the sums' rounding / 1e-5


def test_gradients_of_a_block_against_differences():
    x = lm_layer.inputs(6, 10, 7, 3)
    out, grads = lm_layer.block(lm_layer.Exact(), x)

    def loss(x):
        out, _ = lm_layer.block(lm_layer.Exact(), x)
        return (out["y2"] * x["dy"]).sum() + (out["res2"] * x["dres"]).sum()

    g = np.random.default_rng(2)
    for name, grad in grads.items():
        d = g.standard_normal(grad.shape)
        diff = (loss({**x, name: x[name] + 1e-5 * d}) - loss({**x, name: x[name] - 1e-5 * d})) / 2e-5
        assert abs(diff - (grad * d).sum()) < 1e-6 * max(1, abs(diff)), name   # 1e-10 of the step, 1e-11 of the sums' rounding / 1e-5
