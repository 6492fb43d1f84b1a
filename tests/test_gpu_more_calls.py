"""Calls of the C entry points that the binding does not make: results and codes with pitches of their own, gradients in the place of logits, and calls whose sums go through a
workspace in captured graphs.  What lies between rows, behind them and behind the last one stays as it was."""
import pytest
import torch

pytestmark = pytest.mark.gpu
SENTINEL = 77


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def call(imu, name, *args):
    import ctypes as C
    f = getattr(imu._lib, name)
    f.restype = C.c_int
    def turn(a):
        if a is None:
            return C.c_void_p(None)
        if torch.is_tensor(a):
            return C.c_void_p(a.data_ptr())
        return C.c_int64(a)      # (every integer argument passes in a register of its own; what is an int takes the lower half)
    assert f(*[turn(a) for a in args], C.c_void_p(imu._stream())) == 0


def filled(rows, pitch, dtype):
    return torch.full((rows + 2, pitch), SENTINEL, device="cuda").to(dtype)


def untouched(buf, rows, cols):
    return bool((buf[:rows, cols:].float() == SENTINEL).all()) and bool((buf[rows:].float() == SENTINEL).all())


@pytest.mark.parametrize("m,n,k", [(3, 50, 300), (16, 777, 129), (40, 70, 500), (130, 200, 2048), (700, 523, 384), (2600, 2300, 256), (64, 100, 9000)])
def test_results_with_a_pitch(imu, m, n, k):
    a, b = (imu.imunpack_block8_quantize(torch.randn(r, k, device="cuda"))[0] for r in (m, n))
    for dtype in (torch.float32, torch.bfloat16):
        half = int(dtype == torch.bfloat16)
        want = imu.imunpack_block8_gemm(a, b, dtype)
        for pitch in (n + 5, n + 64):
            out = filled(m, pitch, dtype)
            ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
            call(imu, "imunpack_block8_gemm", a.codes, a.codes.stride(0), a.scales, a.scales.stride(0), 0, b.codes, b.codes.stride(0), b.scales, b.scales.stride(0), 0, m, n, k, None, out, pitch,
                 half, ws, ws.numel())
            assert torch.equal(out[:m, :n], want) and untouched(out, m, n)


@pytest.mark.parametrize("m,n,k", [(5, 60, 200), (100, 200, 640), (700, 523, 1300), (2600, 2300, 384)])
def test_bytes_behind_the_blocks(imu, m, n, k):
    """Nothing is taken from the scales behind a row's blocks: 255 there would make NaN of zeros."""
    a, b = (imu.imunpack_block8_quantize(torch.randn(r, k, device="cuda"))[0] for r in (m, n))
    blocks = -(-k // 128)
    for dtype in (torch.float32, torch.bfloat16):
        want = imu.imunpack_block8_gemm(a, b, dtype)
        scales = [torch.full((len(t.scales) + 1, 32), 255, dtype=torch.uint8, device="cuda") for t in (a, b)]
        for buf, t in zip(scales, (a, b)):
            buf[:-1, :blocks] = t.scales.view(torch.uint8)[:, :blocks]
        out, ws = torch.empty_like(want), torch.empty(64 << 20, dtype=torch.uint8, device="cuda")
        call(imu, "imunpack_block8_gemm", a.codes, a.codes.stride(0), scales[0], 32, 0, b.codes, b.codes.stride(0), scales[1], 32, 0, m, n, k, None, out, n, int(dtype == torch.bfloat16), ws, ws.numel())
        assert torch.equal(out, want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low", [-1e4, -1e5, -1e6, -2.0 ** 20, -1e7, -1e9, -1e10, -1e30, 1e10, 1e30])
def test_logits_of_large_numbers(imu, low, dtype):
    """Rows that a mask's number fills, alone or but for a few.  Log probabilities of elements that the maximum does not outweigh have the size of the spread, which is what their
    tolerance is relative to; l - m is exact or rounded at its own size."""
    vocab = 5000
    x = torch.full((6, vocab), low)
    x[1, 7] += 1.5                     # (what becomes of it is up to the type)
    x[2, 3000:] *= 1 + 2.0 ** -7
    x[3, ::3] *= 1 + 2.0 ** -6
    x[4, 11], x[4, 12] = 0.25, -0.5
    x[5] = low + torch.randn(vocab, generator=torch.Generator().manual_seed(2)) * 2
    x = x.to(dtype)
    tokens = torch.tensor([[0, 7, 11, 12, 3000, 4999]]).expand(6, -1).contiguous()
    got = imu.imunpack_logprobs(x.cuda(), tokens.cuda(), top=8)
    d = x.double() - x.double().amax(1, keepdim=True)
    logs = torch.log(torch.exp(d).sum(1, keepdim=True))
    logp = d - logs
    p = torch.exp(logp)
    h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    near = torch.where(d > -100, d, torch.zeros_like(d)).abs().amax(1)
    want = logp.gather(1, tokens)
    assert ((got.logp.cpu().double() - want).abs() <= 2.0 ** -18 + 2.0 ** -22 * want.abs()).all()
    assert ((got.entropy.cpu().double() - h).abs() <= 2.0 ** -18 * (1 + near)).all()
    lse = x.double().amax(1) + logs[:, 0]
    assert ((got.lse.cpu().double() - lse).abs() <= 2.0 ** -18 + 2.0 ** -22 * lse.abs()).all()
    gp, gh = torch.randn(6, 6), torch.randn(6)
    gl = imu.imunpack_logprobs_backward(x.cuda(), tokens.cuda(), got, gp.cuda(), gh.cuda(), None).cpu().double()
    g = -p * gp.double().sum(1, keepdim=True) - gh.double()[:, None] * torch.where(p > 0, p * (logp + h[:, None]), torch.zeros_like(p))
    g.scatter_add_(1, tokens, gp.double())
    size = 2.0 ** -17 * (p * (gp.abs().double().sum(1, keepdim=True) + gh.abs().double()[:, None] * (10 + 2 * near[:, None])) + 1e-3 * gp.abs().double().amax())
    assert ((gl - g).abs() <= size + g.abs() * torch.finfo(dtype).eps).all()


@pytest.mark.parametrize("rows,cols", [(1, 5), (130, 300), (257, 128)])
def test_codes_with_a_pitch(imu, rows, cols):
    x = torch.randn(rows, cols, device="cuda")
    q, t = imu.imunpack_block8_quantize(x, turned=True)
    wide, tall, kb, rb = -(-cols // 128) * 128, -(-rows // 128) * 128, -(-cols // 128), -(-rows // 128)
    bufs = [torch.full(shape, SENTINEL, dtype=torch.uint8, device="cuda") for shape in ((rows + 2, wide + 48), (rows + 2, 64), (cols + 2, tall + 16), (cols + 2, 32))]
    call(imu, "imunpack_block8_quantize", x, cols, rows, cols, 0, 0, 0, bufs[0], wide + 48, bufs[1], 64, bufs[2], tall + 16, bufs[3], 32)
    as_bytes = lambda v: v.view(torch.uint8)  # noqa: E731
    for buf, want, r, c in ((bufs[0], q.codes, rows, wide), (bufs[1], q.scales, rows, kb), (bufs[2], t.codes, cols, tall), (bufs[3], t.scales, cols, rb)):
        assert torch.equal(buf[:r, :c], as_bytes(want)[:, :c]) and untouched(buf, r, c)
    back = torch.full((cols + 2, tall + 32), SENTINEL, dtype=torch.uint8, device="cuda")
    powers = torch.full((cols + 2, 16), SENTINEL, dtype=torch.uint8, device="cuda")
    call(imu, "imunpack_block8_turn", bufs[0], wide + 48, bufs[1], 64, rows, cols, 0, back, tall + 32, powers, 16)
    want = imu.imunpack_block8_turn(q)
    assert torch.equal(back[:cols, :tall], as_bytes(want.codes)) and untouched(back, cols, tall) and untouched(powers, cols, rb)
    out = filled(rows, cols + 3, torch.float32)
    call(imu, "imunpack_block8_values", bufs[0], wide + 48, bufs[1], 64, rows, cols, 0, out, cols + 3, 0)
    assert torch.equal(out[:rows, :cols], q.values()) and untouched(out, rows, cols)


def test_activations_with_pitches(imu):
    rows, cols = 37, 201
    u = torch.randn(rows, 2 * cols + 9, device="cuda")
    view = u[:, : 2 * cols]
    y, codes, kept = imu.imunpack_act8(view, "gelu", True, quantize=True)
    out, q, qs = filled(rows, cols + 7, torch.float32), torch.full((rows + 2, 320), SENTINEL, dtype=torch.uint8, device="cuda"), torch.full((rows + 2, 16), SENTINEL, dtype=torch.uint8, device="cuda")
    k, k2, ks, k2s = (torch.full((rows + 2, w), SENTINEL, dtype=torch.uint8, device="cuda") for w in (272, 272, 48, 48))
    call(imu, "imunpack_act8", u, 2 * cols + 9, rows, cols, 0, 0, 1, out, cols + 7, q, 320, qs, 16, k, k2, 272, ks, k2s, 48)
    assert torch.equal(out[:rows, :cols], y) and untouched(out, rows, cols)
    for buf, want, c in ((q, codes.codes, 256), (qs, codes.scales, 2), (k, kept[0].codes, 256), (ks, kept[0].scales, 2), (k2, kept[1].codes, 256), (k2s, kept[1].scales, 2)):
        assert torch.equal(buf[:rows, :c], want.view(torch.uint8)[:, :c]) and untouched(buf, rows, c)
    gu = filled(rows, 2 * cols + 1, torch.float32)
    call(imu, "imunpack_act8_backward", out, cols + 7, rows, cols, 0, 0, 1, k, k2, 272, ks, k2s, 48, gu, 2 * cols + 1)
    assert torch.equal(gu[:rows, : 2 * cols], imu.imunpack_act8_backward(y, kept, "gelu", True)) and untouched(gu, rows, 2 * cols)


@pytest.mark.parametrize("rows,vocab", [(3, 1000), (5, 40001), (2100, 333)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradient_in_the_place_of_logits(imu, rows, vocab, dtype):
    """Tokens' logits are read before they are overwritten, whichever part of the row they lie in."""
    buf = filled(rows, vocab + 11, dtype)
    buf[:rows, :vocab] = (torch.randn(rows, vocab, device="cuda") * 2).to(dtype)
    x = buf[:rows, :vocab].contiguous()
    t = torch.randint(0, vocab, (rows, 3), device="cuda")
    t[:, 2] = t[:, 0]
    got = imu.imunpack_logprobs(buf[:rows, :vocab], t, top=4)
    gp, gh, gt = torch.randn(rows, 3, device="cuda"), torch.randn(rows, device="cuda"), torch.randn(rows, 4, device="cuda")
    want = imu.imunpack_logprobs_backward(x, t, got, gp, gh, gt)
    half = int(dtype == torch.bfloat16)
    call(imu, "imunpack_logprobs_backward", buf, vocab + 11, rows, vocab, half, t, 3, -100, 4, got.top_index, got.stats, got.entropy, gp, gh, gt, buf, vocab + 11)
    assert torch.equal(buf[:rows, :vocab], want) and untouched(buf, rows, vocab)


def test_sums_in_parts_in_graphs(imu):
    """Products and log probabilities whose parts meet in a workspace: two graphs in turn, with eager calls of the same between them."""
    a = imu.imunpack_block8_quantize(torch.randn(64, 4096, device="cuda"))[0]
    b = imu.imunpack_block8_quantize(torch.randn(512, 4096, device="cuda"))[0]
    assert imu.imunpack_block8_gemm(a, b).shape == (64, 512)
    logits, tokens = torch.randn(4, 50000, device="cuda"), torch.randint(0, 50000, (4, 2), device="cuda")
    x = torch.randn(64, 4096, device="cuda")
    def step():
        q, _ = imu.imunpack_block8_quantize(x)
        r = imu.imunpack_logprobs(logits, tokens, top=9)
        return imu.imunpack_block8_gemm(q, b), imu.imunpack_block8_gemm(q, b, torch.bfloat16), r.logp, r.entropy, r.top_index, imu.imunpack_logprobs_backward(logits, tokens, r, r.logp)
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for k in range(6):
        x.normal_()
        logits.normal_()
        step()
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(out, step()))
        torch.cuda.synchronize()


def test_two_streams_at_once(imu):
    x = [torch.randn(300, 1000, device="cuda") for _ in range(2)]
    w = imu.imunpack_block8_quantize(torch.randn(700, 1000, device="cuda"))[0]
    def chain(v):
        q, t = imu.imunpack_block8_quantize(v, turned=True)
        y = imu.imunpack_block8_gemm(q, w)
        r = imu.imunpack_logprobs(y, top=7)
        return y, r.lse, r.top_index, imu.imunpack_block8_gemm(t, imu.imunpack_block8_turn(q))
    want = [chain(v) for v in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        got = []
        for s, v in zip(streams, x):
            with torch.cuda.stream(s):
                got.append(chain(v))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, e in zip(got, want) for a, b in zip(g, e))
