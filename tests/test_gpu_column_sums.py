"""Sums of columns against binary64, and what they are for: gradients of biases, also of layers whose passes are replayed from a graph.

Tolerance: an element passes at most rows / 16 + 64 additions (a thread's own of a part, sixteen groups, the parts', sixteen groups again), each off by 2^-24 of a partial sum of magnitudes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def check(got, x):
    x = x.double().reshape(-1, x.shape[-1])
    assert got.dtype == torch.float32 and got.shape == x.shape[1:]
    assert ((got.double() - x.sum(0)).abs() <= (x.shape[0] / 16 + 64) * 2.0 ** -24 * x.abs().sum(0)).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 1000), (2, 3), (15, 64), (16, 65), (17, 127), (63, 129), (127, 40), (128, 40), (129, 256), (1000, 777), (4097, 63), (5000, 1), (12608, 768), (300, 40001),
                                       (100003, 8)])
def test_sums(imu, rows, cols, dtype):
    x = torch.randn(rows, cols, device="cuda", generator=torch.Generator("cuda").manual_seed(rows + cols)).to(dtype)
    got = imu.imunpack_column_sums(x)
    check(got, x)
    assert torch.equal(got, imu.imunpack_column_sums(x))


def test_layouts(imu):
    wide = torch.randn(700, 131, device="cuda")
    check(imu.imunpack_column_sums(wide[:, 1:100]), wide[:, 1:100])
    check(imu.imunpack_column_sums(wide[::3, 3:7]), wide[::3, 3:7])
    check(imu.imunpack_column_sums(wide.t()), wide.t())
    check(imu.imunpack_column_sums(wide[:1].expand(500, -1)), wide[:1].expand(500, -1))
    check(imu.imunpack_column_sums(wide.view(7, 100, 131)), wide)
    check(imu.imunpack_column_sums(wide[5]), wide[5:6])
    assert torch.equal(imu.imunpack_column_sums(wide[:0]), torch.zeros(131, device="cuda"))
    odd = wide.clone()
    odd[3, 5], odd[600, 6], odd[10, 7], odd[650, 7] = float("inf"), float("nan"), float("inf"), -float("inf")
    got = imu.imunpack_column_sums(odd)
    assert torch.isposinf(got[5]) and torch.isnan(got[6]) and torch.isnan(got[7]) and int(torch.isfinite(got).sum()) == 128
    for bad in (wide.half(), wide.cpu(), torch.empty(5, 0, device="cuda")):
        with pytest.raises((ValueError, TypeError)):
            imu.imunpack_column_sums(bad)


LAYERS = [("linear", 4096, 256, 512, torch.float32), ("linear", 130, 64, 70, torch.bfloat16), ("mlp", 2048, 256, 1024, torch.float32), ("gated", 2048, 256, 512, torch.bfloat16), ("gated", 77, 96, 200, torch.float32)]


@pytest.mark.parametrize("kind,rows,d,hidden,dtype", LAYERS)
def test_passes_in_a_graph(imu, kind, rows, d, hidden, dtype):
    """Both passes of a layer with biases in two graphs, which take turns with eager steps on other data; every replay's gradients are an eager step's, bit by bit."""
    from paper_2403_07339_amd.block8 import Block8Linear, Block8MLP
    torch.manual_seed(1)
    layer = Block8Linear(d, hidden, device="cuda", dtype=dtype) if kind == "linear" else Block8MLP(d, hidden, "silu" if kind == "gated" else "gelu", kind == "gated", device="cuda", dtype=dtype)
    x = torch.randn(rows, d, device="cuda").to(dtype).requires_grad_()
    gy = torch.randn(rows, hidden if kind == "linear" else d, device="cuda").to(dtype)
    leaves = [x, *layer.parameters()]
    step = lambda: (lambda y: (y.detach(), *torch.autograd.grad(y, leaves, gy)))(layer(x))  # noqa: E731
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for k in range(8):
        with torch.no_grad():
            x.normal_()
            gy.normal_()
        want = step()
        torch.cuda.synchronize()
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(out, want)), k
        with torch.no_grad():
            x.normal_()
        step()


def test_layers_without_features_are_refused(imu):
    from paper_2403_07339_amd.block8 import block8_linear, block8_mlp
    e = lambda *s: torch.empty(*s, device="cuda")  # noqa: E731
    for x, w in ((e(3, 0), e(5, 0)), (e(3, 4), e(0, 4))):
        with pytest.raises(ValueError):
            block8_linear(x, w)
    for x, w1, w2 in ((e(3, 0), e(8, 0), e(2, 8)), (e(3, 4), e(0, 4), e(2, 0)), (e(3, 4), e(8, 4), e(0, 8))):
        with pytest.raises(ValueError):
            block8_mlp(x, w1, w2)
