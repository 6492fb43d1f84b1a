"""Several tensors brought into 8 bits by one launch: bit by bit what the calls for one give."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def same(a, b):
    if a is None or b is None:
        return a is b
    blocks = -(-a.cols // 128)
    raw = lambda v: v.view(torch.uint8)  # noqa: E731
    return a.cols == b.cols and a.codes.dtype == b.codes.dtype and torch.equal(raw(a.codes), raw(b.codes)) and torch.equal(raw(a.scales)[:, :blocks], raw(b.scales)[:, :blocks])


def one(imu, w, format):
    if isinstance(w, imu.Blocks8):
        return None, imu.imunpack_block8_turn(w)
    x, square, lying, turned = w
    return imu.imunpack_block8_quantize(x, format, square, turned, lying)


def tensor(rows, cols, dtype=torch.float32, seed=0):
    g = torch.Generator("cuda").manual_seed(seed + rows + cols)
    return (torch.randn(rows, cols, device="cuda", generator=g) * torch.exp2(torch.randint(-9, 9, (rows, 1), device="cuda", generator=g).float())).to(dtype)


@pytest.mark.parametrize("format", ["e4m3", "e5m2"])
@pytest.mark.parametrize("shapes", [[(1, 1), (1, 1)], [(197, 256), (1000, 256)], [(3, 129), (300, 7), (128, 128), (129, 1000)], [(2000, 1), (1, 2000), (513, 640)], [(12608, 768), (768, 768)], [(5, 40000), (4000, 500)]])
def test_as_one_by_one(imu, shapes, format):
    kinds = [(False, True, False), (True, True, True), (False, True, True), (False, False, True), (True, False, True), (True, True, False), "turn"]
    for shift in range(len(kinds)):
        wanted = []
        for k, (rows, cols) in enumerate(shapes):
            x, kind = tensor(rows, cols, [torch.float32, torch.bfloat16][(k + shift) % 2], k), kinds[(k + shift) % len(kinds)]
            wanted.append(imu.imunpack_block8_quantize(x, format)[0] if kind == "turn" else (x, *kind))
        for got, w in zip(imu.imunpack_block8_many(*wanted, format=format), wanted):
            want = one(imu, w, format)
            assert same(got[0], want[0]) and same(got[1], want[1])


def test_views_and_empty_ones_and_more_than_a_launch(imu):
    base = tensor(400, 600)
    wanted = [(base[::2, 3:500], False, True, True), (base.t(), True, True, False), (base[:0], False, True, False), (base.view(4, 100, 600), False, True, False)]
    got = imu.imunpack_block8_many(*wanted)
    for (q, t), w in zip(got, wanted):
        want = one(imu, w, "e4m3")
        assert same(q, want[0]) and same(t, want[1])
    assert got[2][0].codes.shape == (0, 640)
    assert same(imu.imunpack_block8_many((base, False, True, False))[0][0], imu.imunpack_block8_quantize(base)[0])
    rows = (1 << 26) + 1     # more blocks than one launch takes, beside a small one
    long = torch.ones(rows, 1, device="cuda", dtype=torch.bfloat16)
    (q, _), (s, _) = imu.imunpack_block8_many((long, False, True, False), (base, False, True, False))
    assert same(s, imu.imunpack_block8_quantize(base)[0]) and bool((q.values(torch.bfloat16)[-1000:] == 1).all())
    del q
    torch.cuda.empty_cache()


def test_in_a_graph(imu):
    x, w = tensor(197, 256), tensor(1000, 256, torch.bfloat16)
    kept = imu.imunpack_block8_quantize(tensor(300, 200))[0]
    step = lambda: imu.imunpack_block8_many((x, False, True, True), (w, True, True, True), kept)  # noqa: E731
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(4):
        x.normal_()
        w.normal_()
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(same(a, b) for got, e in zip(out, want) for a, b in zip(got, e))


def test_refusals(imu):
    x = tensor(10, 200)
    q = imu.imunpack_block8_quantize(x)[0]
    good = (x, False, True, False)
    for bad in ((x.half(), False, True, False), (x.cpu(), False, True, False), (x[:, :0], False, True, False), (x, False, False, False), (x[:0], False, False, True), imu.Blocks8(q.codes, q.scales, 300),
                imu.Blocks8(q.codes, q.scales[:5], 200), imu.imunpack_block8_quantize(x, "e5m2")[0], (x, False, True)):
        with pytest.raises(ValueError):
            imu.imunpack_block8_many(good, bad)
        with pytest.raises(ValueError):
            imu.imunpack_block8_many(bad, good)
    for count in (0, 5):
        with pytest.raises(ValueError):
            imu.imunpack_block8_many(*[good] * count)
    with pytest.raises(ValueError):
        imu.imunpack_block8_many(good, format="e3m4")
