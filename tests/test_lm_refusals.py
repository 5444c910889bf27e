"""What the calls of the language-model layer refuse before any launch (CPU)."""
import pytest
import torch

NULL, SHAPE, WS, VALUE = -1, -2, -5, -7


@pytest.fixture(scope="module")
def q8t():
    from test_abi import _lib_path
    _lib_path()
    import paper_1805_11046_amd as m
    return m


@pytest.fixture(scope="module")
def L(q8t):
    return q8t.binding._lib


def test_fp8_quantize(L):
    f = lambda x=16, type=0, R=4, C=4, fmt=0, q=16, s=16, qt=None, st=None: L.q8t_fp8_quantize(x, type, R, C, fmt, 0, 0, 0, None, q, s, qt, st, None)   # noqa: E731
    assert f(x=None) == NULL and f(q=None) == NULL and f(s=None) == NULL and f(qt=16) == NULL and f(st=16) == NULL
    assert f(type=2) == VALUE and f(type=-1) == VALUE and f(fmt=2) == VALUE and f(fmt=-1) == VALUE
    assert f(R=-1) == SHAPE and f(C=-1) == SHAPE and f(R=1 << 31, C=1) == SHAPE and f(R=1, C=1 << 31) == SHAPE
    assert f(R=1 << 18, C=(1 << 16) + 1) == SHAPE and f(R=1 << 28, C=1) == SHAPE and f(R=1, C=1 << 28) == SHAPE
    assert f(q=8) == SHAPE and f(qt=8, st=16) == SHAPE
    assert f(x=None, q=None, s=None, R=0) == 0 and f(x=None, q=None, s=None, C=0) == 0


def test_fp8_gemm(L):
    def f(a=16, sa=16, fa=0, b=16, sb=16, fb=0, M=4, N=4, K=4, out=16, type=0):
        return L.q8t_fp8_gemm(a, sa, fa, b, sb, fb, M, N, K, out, type, None, None)
    assert all(f(**{k: None}) == NULL for k in ("a", "sa", "b", "sb", "out"))
    assert f(fa=2) == VALUE and f(fb=-1) == VALUE and f(type=2) == VALUE
    assert f(M=-1) == SHAPE and f(N=-1) == SHAPE and f(K=0) == SHAPE and f(K=-5) == SHAPE and f(K=(1 << 23) + 1) == SHAPE and f(M=1 << 19, N=(1 << 17) + 1) == SHAPE and f(M=(1 << 22) + 1) == SHAPE
    assert f(a=8) == SHAPE and f(b=8) == SHAPE and f(sa=2) == SHAPE and f(sb=2) == SHAPE
    assert f(M=0, a=None, out=None) == 0 and f(N=0) == 0
    assert L.q8t_fp8_gemm_workspace_size(0, 4, 4) == 0 and L.q8t_fp8_gemm_workspace_size(-1, 4, 4) == 0


def test_residual_norm(L):
    def f(res=16, h=16, wp=16, gate=16, G=2, wq=16, type=0, T=4, D=8, rs=1.0, p=0.0, r=16, y=16, q=None, s=None):
        return L.q8t_residual_norm_fwd(res, h, wp, gate, G, wq, type, T, D, 1e-6, rs, 1.0, p, 0, None, r, y, 16, q, s, None)
    assert f(res=None) == NULL and f(r=None) == NULL and f(y=None) == NULL and f(q=16) == NULL and f(s=16) == NULL and f(wq=None) == NULL
    assert f(type=2) == VALUE and f(p=-0.1) == VALUE and f(p=1.1) == VALUE and f(p=float("nan")) == VALUE
    assert f(h=None) == VALUE and f(h=None, wp=None, gate=None, G=0, rs=2.0) == VALUE and f(h=None, wp=None, gate=None, G=0, p=0.5) == VALUE
    assert f(T=-1) == SHAPE and f(D=0) == SHAPE and f(D=16385) == SHAPE and f(T=1 << 22) == SHAPE and f(G=3) == SHAPE and f(G=0) == SHAPE
    assert f(gate=None) == SHAPE and f(G=-1) == SHAPE and f(q=8, s=16) == SHAPE
    assert f(h=None, wp=None, gate=None, G=0, wq=None, y=None) == NULL
    assert f(T=0, res=None, r=None) == 0

    def g(dy=16, dro=16, r=16, h=16, st=16, wp=16, gate=16, G=2, wq=16, type=0, T=4, D=8, p=0.0, dres=16, dh=16, dg=16, dwp=16, dwq=16, ws=16):
        return L.q8t_residual_norm_bwd(dy, dro, r, h, st, wp, gate, G, wq, type, T, D, 1.0, 1.0, p, 0, None, dres, dh, dg, dwp, dwq, ws, None)
    for k in ("dy", "r", "st", "dh", "dg", "dwp", "dwq"):
        assert g(**{k: None}) == NULL, k
    assert g(dy=None, dro=None, wq=None, dwq=None) == NULL and g(h=None, dh=None) == VALUE
    assert g(h=None, dh=None, wp=None, dwp=None, gate=None, G=0, dg=None, dres=None) == NULL
    assert g(ws=None) == WS and g(ws=8) == WS and g(type=3) == VALUE and g(p=-1.0) == VALUE and g(G=3) == SHAPE and g(D=0) == SHAPE
    size = L.q8t_residual_norm_bwd_workspace_size
    assert size(0, 8, 0) == 0 and size(4, 0, 0) == 0 and size(4, 8, 3) == 0 and size(4, 8, 2) > 0


@pytest.mark.parametrize("T,groups", [(T, G) for T in (1, 2, 511, 512, 513, 1000, 1024, 1536, 4100, 100000) for G in (0, 1, 2, 3, 5, 7, 500, 512, T)
                                      if G == 0 or T % G == 0])
def test_workspace_of_the_norms_backward_stays_small(L, T, groups):
    # a workgroup a chunk of rows leaves three rows of sums (whole lines): at most about twice 2048 chunks of narrow rows, 512 of wide
    # ones, of one row at least
    for D, most in ((8, 2048), (4096, 512)):
        chunks = L.q8t_residual_norm_bwd_workspace_size(T, D, groups) / (3 * max(D, 32) * 4)
        assert 1 <= chunks <= min(2.2 * most, 2 * T)


def test_dropout(L):
    f = lambda x=16, type=0, n=4, p=0.5, out=16: L.q8t_dropout(x, None, type, n, p, 0, None, out, None)   # noqa: E731
    assert f(x=None) == NULL and f(out=None) == NULL and f(n=-1) == SHAPE and f(n=(1 << 34) + 1) == SHAPE
    assert f(type=5) == VALUE and f(p=-0.5) == VALUE and f(p=1.5) == VALUE and f(p=float("nan")) == VALUE
    assert f(n=0, x=None) == 0


def test_cpu_tensors_and_other_arguments(q8t):
    x, w = torch.zeros(4, 8), torch.zeros(8)
    q, s = torch.zeros(4, 128, dtype=torch.float8_e4m3fn), torch.zeros(4, 4, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    for call in (lambda: q8t.fp8_quantize(x), lambda: q8t.fp8_gemm(q, s, q, s), lambda: q8t.residual_norm_fwd(x, x, w_post=w, w_pre=w),
                 lambda: q8t.residual_norm_bwd(x, x, x, x, x, w_pre=w), lambda: q8t.dropout(x, 0.5)):
        with pytest.raises(ValueError, match="device tensors only"):
            call()
    for call in (lambda: q8t.fp8_quantize([1.0]), lambda: q8t.fp8_gemm(None, s, q, s), lambda: q8t.dropout(3, 0.5)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="fmt is one of"):
        q8t.fp8_quantize(x, "e8m0")
    with pytest.raises(ValueError, match="dtype is one of"):
        q8t.fp8_gemm(q, s, q, s, dtype=torch.float16)
