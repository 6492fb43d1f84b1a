"""Log probabilities, entropy, alternatives and their gradient against the definitions in binary64.

Tolerances.  m + log S: an exponential is within 2^-22 of its value and a term passes fewer than 200 additions on its way (a thread's, the tree's, the parts'; those of a
thread are relative to its own partial sum), so S is within 256 * 2^-24 relative and lse within that of 1 (as log S moves), plus two roundings at the size of lse.  An exponent l - m is rounded at
its own size, which is at most the row's spread: another spread * 2^-24 of the term.  With spreads below 64 that is 2^-18 in all, and 2^-22 of |lse| + |l|.
Entropy: sum p (l - m) has terms of size up to spread, so 2^-18 (1 + spread) covers both its parts.  Gradients: p is within 2^-17 of itself, the sum of given gradients 2^-20 of
its magnitudes; bfloat16 results are rounded by 2^-8 of themselves."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F = torch.float64
IGNORE = -100


@pytest.fixture(scope="module")
def imu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2403_07339_amd import binding
    return binding


def data(rows, vocab, count, dtype, seed=0, spread=2.5):
    g = torch.Generator().manual_seed(seed)
    x = (torch.randn(rows, vocab, generator=g) * spread).to(dtype)
    t = torch.randint(0, vocab, (rows, count), generator=g)
    return x, t


def order(x):
    """Places of a row's logits, largest first, of equals the lowest place first; NaN with -infinity."""
    x = torch.where(torch.isnan(x), torch.full_like(x, -float("inf")), x.double())
    return torch.sort(x, dim=1, descending=True, stable=True).indices


def definition(x, tokens):
    x = x.double()
    m = x.amax(1, keepdim=True)
    none = torch.isneginf(m[:, 0])
    e = torch.exp(x - torch.where(torch.isneginf(m), torch.zeros_like(m), m))
    lse = torch.where(none, m[:, 0], m[:, 0] + torch.log(e.sum(1)))
    logp = torch.where(torch.isneginf(x), x, (x - m) - torch.log(e.sum(1, keepdim=True)))   # (beside the lowest number of a type the logarithm is lost)
    p = torch.exp(logp)
    p[none] = 0.0
    h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    return logp, p, lse, h


def check(imu, x, tokens, top, got):
    logp, p, lse, h = definition(x, tokens)
    finite = torch.where(torch.isinf(x), torch.zeros((), dtype=x.dtype), x).double()
    wide = (finite.amax(1) - finite.amin(1)).clamp_min(1.0)
    tol = 2.0 ** -18 + 2.0 ** -22 * (torch.where(torch.isinf(lse), torch.zeros_like(lse), lse).abs() + finite.abs().amax(1))
    same = lambda a, b, t: (torch.equal(torch.isneginf(a), torch.isneginf(b)) and bool(((a - b).abs() <= t)[torch.isfinite(b)].all()))  # noqa: E731
    assert same(got.lse.cpu().double(), lse, tol)
    assert ((got.entropy.cpu().double() - h).abs() <= 2.0 ** -18 * (1 + wide)).all()
    ok = tokens != IGNORE
    want = torch.where(ok, logp.gather(1, tokens.clamp_min(0)), torch.zeros((), dtype=F))
    assert same(got.logp.cpu().double().view(want.shape), want, tol[:, None].expand_as(want))
    if top:
        index = order(x)[:, :top]
        assert torch.equal(got.top_index.cpu(), index)
        assert same(got.top_logp.cpu().double(), logp.gather(1, index), tol[:, None].expand(-1, top))
    return logp, p, lse, h


def check_grad(imu, x, tokens, top, got, gp, gh, gt, gl, dtype):
    logp, p, lse, h = definition(x, tokens)
    none = torch.isneginf(lse)
    ok = (tokens != IGNORE)
    w = torch.zeros_like(logp)
    total, size = torch.zeros(x.shape[0], dtype=F), torch.zeros(x.shape[0], dtype=F)
    if gp is not None:
        g = gp.double() * ok
        w.scatter_add_(1, tokens.clamp_min(0), g)
        total += g.sum(1)
        size += g.abs().sum(1)
    if gt is not None:
        w.scatter_add_(1, order(x)[:, :top], gt.double())
        total += gt.double().sum(1)
        size += gt.double().abs().sum(1)
    want = w - p * total[:, None]
    bound = 2.0 ** -20 * w.abs() + 2.0 ** -17 * p * size[:, None]
    if gh is not None:
        d = torch.where(p > 0, logp + h[:, None], torch.zeros_like(p))
        want -= gh.double()[:, None] * p * d
        bound += 2.0 ** -17 * gh.double().abs()[:, None] * p * (d.abs() + logp.abs().nan_to_num(0, 0, 0) + h.abs()[:, None] + 1)
    want[none] = 0.0
    bound[none] = 0.0
    step = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24
    assert gl.dtype == dtype and gl.shape == x.shape
    off = (gl.cpu().double() - want).abs()
    assert (off <= bound + step * want.abs() + 2.0 ** -120).all(), (off - bound - step * want.abs()).max()


SIZES = [(1, 1, 1), (1, 2, 1), (3, 63, 2), (2, 64, 1), (5, 65, 3), (4, 255, 1), (3, 1000, 4), (7, 1031, 1), (2, 4097, 7), (16, 32000, 1), (3, 50265, 4), (2, 128000, 1), (300, 777, 2), (1, 262147, 3)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,count", SIZES)
def test_forward_and_backward(imu, rows, vocab, count, dtype):
    x, t = data(rows, vocab, count, dtype, rows + vocab)
    if rows > 2:
        t[1, 0] = IGNORE
    g = torch.Generator().manual_seed(5)
    dev, tok = x.cuda(), t.cuda()
    for top in sorted({0, 1, min(5, vocab), min(20, vocab), min(64, vocab)}):
        got = imu.imunpack_logprobs(dev, tok, top=top, ignore_index=IGNORE)
        assert (got.top_logp is None) == (top == 0)
        check(imu, x, t, top, got)
    gp, gh, gt = torch.randn(rows, count, generator=g), torch.randn(rows, generator=g), torch.randn(rows, top, generator=g)
    again = imu.imunpack_logprobs(dev, tok, top=top, ignore_index=IGNORE)
    assert torch.equal(again.lse, got.lse) and torch.equal(again.entropy, got.entropy)
    for a, b, c in ((gp, gh, gt), (gp, None, None), (None, gh, None), (None, None, gt)):
        gl = imu.imunpack_logprobs_backward(dev, tok, got, *(None if v is None else v.cuda() for v in (a, b, c)), ignore_index=IGNORE)
        check_grad(imu, x, t, top, got, a, b, c, gl, dtype)
        assert torch.equal(gl, imu.imunpack_logprobs_backward(dev, tok, got, *(None if v is None else v.cuda() for v in (a, b, c)), ignore_index=IGNORE))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("kind", ["up", "down", "level", "few", "steps", "peaks", "lowest", "far", "mask", "late"])
@pytest.mark.parametrize("vocab", [70, 1500, 20011])
def test_orders_and_masks(imu, vocab, kind, dtype):
    """Rows in which every place beats the ones before it or none does, equal rows, few different values, all but a few masked, logits of the type's lowest value."""
    rows, n = 3, torch.arange(vocab, dtype=torch.float32)
    low = torch.finfo(dtype).min
    x = {"up": n / vocab * 30, "down": -n / vocab * 30, "level": torch.full((vocab,), 3.25), "few": (n % 7), "steps": torch.floor(n / 64) / vocab * 500,
         "peaks": torch.where(n % 64 == 5, n / vocab * 20, -n / vocab), "lowest": torch.where(n % 3 == 0, torch.full_like(n, low), n % 11), "far": n * 0 + low,
         "mask": torch.where(n % 97 == 13, n % 5, torch.full_like(n, -float("inf"))), "late": torch.where(n >= vocab - 3, n * 0 + 1, torch.full_like(n, -float("inf")))}[kind]
    x = torch.stack([x, x.flip(0), torch.roll(x, vocab // 3)]).to(dtype)
    t = torch.tensor([[0, vocab - 1, vocab // 2]] * rows)
    top = 64
    got = imu.imunpack_logprobs(x.cuda(), t.cuda(), top=top)
    logp, p, lse, h = definition(x, t)
    index = order(x)[:, :top]
    assert torch.equal(got.top_index.cpu(), index)
    if kind in ("lowest", "far"):   # a spread of 3e38: entropy and probabilities all the same
        assert ((got.entropy.cpu().double() - h).abs() <= 2.0 ** -18 * (1 + 16)).all()
        live = torch.where(x.double() > low, p, torch.zeros_like(p)) if kind == "lowest" else p
        assert ((torch.exp(got.top_logp.cpu().double()) - live.gather(1, index)).abs() <= 2.0 ** -17).all()
    else:
        check(imu, x, t, top, got)
    g = torch.Generator().manual_seed(vocab)
    gp, gh, gt = torch.randn(rows, 3, generator=g), torch.randn(rows, generator=g), torch.randn(rows, top, generator=g)
    gl = imu.imunpack_logprobs_backward(x.cuda(), t.cuda(), got, gp.cuda(), gh.cuda(), gt.cuda())
    if kind not in ("lowest", "far"):
        check_grad(imu, x, t, top, got, gp, gh, gt, gl, dtype)
    else:
        assert torch.isfinite(gl).all()


def test_a_row_that_a_mask_leaves_empty(imu):
    x, t = data(4, 500, 2, torch.float32, 3)
    x[1] = -float("inf")
    t[2, 1] = 499
    got = imu.imunpack_logprobs(x.cuda(), t.cuda(), top=7)
    check(imu, x, t, 7, got)
    assert float(got.entropy[1]) == 0.0 and torch.isneginf(got.logp[1]).all() and torch.isneginf(got.top_logp[1]).all()
    assert got.top_index[1].tolist() == list(range(7))
    gl = imu.imunpack_logprobs_backward(x.cuda(), t.cuda(), got, torch.ones(4, 2).cuda(), torch.ones(4).cuda(), torch.ones(4, 7).cuda())
    assert not gl[1].any() and torch.isfinite(gl).all()


def test_nan_and_infinity_stay_in_their_row(imu):
    x, t = data(5, 3000, 1, torch.float32, 8)
    clean = imu.imunpack_logprobs(x.cuda(), t.cuda(), top=4)
    y = x.clone()
    y[1, 7], y[3, 2999] = float("nan"), float("inf")
    got = imu.imunpack_logprobs(y.cuda(), t.cuda(), top=4)
    for k in (1, 3):
        assert torch.isnan(got.lse[k]) and torch.isnan(got.entropy[k]) and torch.isnan(got.logp[k]).all() and torch.isnan(got.top_logp[k]).all()
    assert torch.equal(got.top_index.cpu(), order(y)[:, :4])
    rest = [0, 2, 4]
    assert torch.equal(got.lse[rest], clean.lse[rest]) and torch.equal(got.logp[rest], clean.logp[rest]) and torch.equal(got.entropy[rest], clean.entropy[rest])
    gl = imu.imunpack_logprobs_backward(y.cuda(), t.cuda(), got, torch.ones(5, 1).cuda(), torch.ones(5).cuda())
    assert torch.isnan(gl[[1, 3]]).any(1).all() and torch.isfinite(gl[rest]).all()


def test_tokens_twice_ignored_and_outside(imu):
    x, _ = data(3, 900, 1, torch.float32, 4)
    t = torch.tensor([[5, 5, 899, 5], [IGNORE, 0, 900, -1], [IGNORE] * 4])
    got = imu.imunpack_logprobs(x.cuda(), t.cuda(), top=3)
    logp = definition(x, t)[0]
    assert torch.equal(got.logp[0, 0], got.logp[0, 1]) and torch.equal(got.logp[2], torch.zeros(4).cuda())
    assert float(got.logp[1, 0]) == 0.0 and torch.isnan(got.logp[1, 2:]).all()
    assert abs(float(got.logp[1, 1]) - float(logp[1, 0])) <= 2.0 ** -17
    gp = torch.randn(3, 4)
    gl = imu.imunpack_logprobs_backward(x.cuda(), t.cuda(), got, gp.cuda())
    g = gp.clone()
    g[1, [0, 2, 3]] = 0.0
    check_grad(imu, x, torch.tensor([[5, 5, 899, 5], [0, 0, 0, 0], [IGNORE] * 4]), 3, got, g, None, None, gl, torch.float32)
    none = imu.imunpack_logprobs(x.cuda(), top=2, want_entropy=False)
    assert none.logp is None and none.entropy is None and torch.equal(none.lse, got.lse) and torch.equal(none.top_index, got.top_index[:, :2])


def test_layouts_streams_and_graphs(imu):
    base, t = data(40, 2000, 2, torch.bfloat16, 6)
    base, t = base.cuda(), t.cuda()
    want = imu.imunpack_logprobs(base[:20, 3:1500].contiguous(), t[:20] % 1497, top=9)
    got = imu.imunpack_logprobs(base[:20, 3:1500], t[:20] % 1497, top=9)
    assert torch.equal(got.lse, want.lse) and torch.equal(got.top_index, want.top_index) and torch.equal(got.logp, want.logp)
    gh = torch.randn(20).cuda()
    assert torch.equal(imu.imunpack_logprobs_backward(base[:20, 3:1500], t[:20] % 1497, got, None, gh), imu.imunpack_logprobs_backward(base[:20, 3:1500].contiguous(), t[:20] % 1497, want, None, gh))
    turned = imu.imunpack_logprobs(base.t()[:, :30], top=1)
    assert torch.equal(turned.top_index[:, 0].cpu(), order(base.t()[:, :30].float().cpu())[:, 0])
    deep = imu.imunpack_logprobs(base.view(4, 10, 2000), t.view(4, 10, 2), top=2)
    flat = imu.imunpack_logprobs(base, t, top=2)
    assert deep.logp.shape == (4, 10, 2) and deep.lse.shape == (4, 10) and deep.top_index.shape == (4, 10, 2) and torch.equal(deep.logp.view(40, 2), flat.logp)
    single = imu.imunpack_logprobs(base[0], t[0, 0], top=1)
    assert single.logp.shape == () and torch.equal(single.logp, flat.logp[0, 0])
    empty = imu.imunpack_logprobs(base[:0], t[:0], top=2)
    assert empty.logp.shape == (0, 2) and imu.imunpack_logprobs_backward(base[:0], t[:0], empty, torch.zeros(0, 2).cuda()).shape == (0, 2000)
    x = base.clone()
    gp = torch.randn(40, 2).cuda()
    def step():
        r = imu.imunpack_logprobs(x, t, top=5)
        return r.logp, r.entropy, r.top_index, imu.imunpack_logprobs_backward(x, t, r, gp, r.entropy)
    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):   # two graphs, in turn, with eager calls between them
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for k in range(6):
        x.copy_(base.roll(k, 1) * (1 + k % 2))
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, step()))


def test_gradient_against_differences(imu):
    """logp and entropy of rows in binary64, moved along a direction."""
    x, t = data(6, 300, 2, torch.float32, 9)
    got = imu.imunpack_logprobs(x.cuda(), t.cuda(), top=3)
    gp, gh = torch.randn(6, 2), torch.randn(6)
    gl = imu.imunpack_logprobs_backward(x.cuda(), t.cuda(), got, gp.cuda(), gh.cuda()).cpu().double()
    way = torch.randn(6, 300, dtype=F)
    def value(s):
        logp = torch.log_softmax(x.double() + s * way, 1)
        return (gp.double() * logp.gather(1, t)).sum(1) - gh.double() * (logp.exp() * logp).sum(1)
    d = 1e-4
    slope = (value(d) - value(-d)) / (2 * d)   # (d^2 / 6 times a third derivative of some hundreds at most: 1e-6)
    assert (((gl * way).sum(1) - slope).abs() <= 2e-5 + 2.0 ** -17 * (gp.abs().sum(1).double() + 20 * gh.abs().double())).all()


def test_refusals(imu):
    x, t = data(4, 50, 1, torch.float32)
    x, t = x.cuda(), t.cuda()
    for call in (lambda: imu.imunpack_logprobs(x.half(), t), lambda: imu.imunpack_logprobs(x.cpu(), t), lambda: imu.imunpack_logprobs(x, t.int()), lambda: imu.imunpack_logprobs(x, t[:3]),
                 lambda: imu.imunpack_logprobs(x, t.cpu()), lambda: imu.imunpack_logprobs(x, t, top=51), lambda: imu.imunpack_logprobs(x, t, top=-1), lambda: imu.imunpack_logprobs(x[:, :0], t)):
        with pytest.raises(ValueError):
            call()
    got = imu.imunpack_logprobs(x, t, top=2)
    wide = imu.imunpack_logprobs(torch.randn(2, 100).cuda(), top=2)
    for call in (lambda: imu.imunpack_logprobs_backward(x, t, got, torch.ones(3, 1).cuda()), lambda: imu.imunpack_logprobs_backward(x, None, got, torch.ones(4, 1).cuda()),
                 lambda: imu.imunpack_logprobs_backward(x, t, got, None, torch.ones(4).cuda().half()), lambda: imu.imunpack_logprobs_backward(x, t, wide, torch.ones(4, 1).cuda()),
                 lambda: imu.imunpack_logprobs_backward(x, t, got, g_top=torch.ones(4, 3).cuda()),
                 lambda: imu.imunpack_logprobs_backward(x, t, imu.imunpack_logprobs(x, t, want_entropy=False), g_entropy=torch.ones(4).cuda())):
        with pytest.raises(ValueError):
            call()
    big = torch.randn(2, 3000).cuda()
    with pytest.raises(ValueError):
        imu.imunpack_logprobs(big, top=65)
    with pytest.raises(imu.ImunpackError):
        imu.imunpack_logprobs(big, torch.zeros(2, 1025, dtype=torch.int64).cuda())
