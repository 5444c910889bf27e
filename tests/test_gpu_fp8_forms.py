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


@pytest.mark.parametrize("M,N,K", [(70, 300, 8192), (300, 520, 4097)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_streams_and_graphs_of_sliced_products(M, N, K, dtype):
    # the partial sums of the slices lie in scratch memory: two streams' calls, a captured one and an eager one have their own
    q8t = require_gpu()
    import torch
    assert q8t.binding._lib.q8t_fp8_gemm_workspace_size(M, N, K) > 0
    ops = [(_operand(M, K, "e4m3", 10 + i), _operand(N, K, "e5m2", 20 + i)) for i in range(2)]
    call = lambda i: q8t.fp8_gemm(*ops[i][0][0], *ops[i][1][0], dtype=getattr(torch, dtype))   # noqa: E731
    want = [(va @ vb.T).to(getattr(torch, dtype)).to("cuda:0") for (_, va), (_, vb) in ops]
    assert not torch.equal(want[0], want[1])
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(8):
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
    for _ in range(4):
        for i, (g, out) in enumerate(graphs):
            out.zero_()
            g.replay()
            eager = call(1 - i)
            torch.cuda.synchronize()
            assert torch.equal(out, want[i]) and torch.equal(eager, want[1 - i])
    # both graphs at once, on two streams
    for out in (o for _, o in graphs):
        out.zero_()
    for s, (g, _) in zip(streams, graphs):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out, w) for (_, out), w in zip(graphs, want))
