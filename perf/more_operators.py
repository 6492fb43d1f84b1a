"""Products in 8-bit floating point, activations kept in 8 bits and log probabilities, as cases that can be timed.

``listed()`` names the cases, ``draw()`` gives others of the same ranges, ``prepare()`` makes what a program holds before the
call, ``run()`` is one pass: with ``own`` through the framework's entry points, else in plain form, elementary torch
operations in 32 bits rounded once at the end.  ``exact()`` is the definition in 64 bits.

A tensor in 8 bits is codes (e4m3, or e5m2) with a power of two for every 128 of a row, or for every 128 x 128 (weights): the smallest
that brings the block's largest magnitude to the type's largest.

Kinds:
  product   A B^T (+ bias) of two such tensors: serving, the weights laid out beforehand
  linear    a training step of a linear layer: x, w and gy become 8 bits, x is kept that way for the gradient of w
  act       GELU or SiLU, gated or not, whose input is kept in 8 bits for the backward pass
  logprobs  log probabilities of given tokens, entropy and top alternatives of a row of logits; with the gradient where it trains
"""
from __future__ import annotations

import math

import torch

own = False

BLOCK = 128
IGNORE = -100
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4.0, "bf16": 2.0}
CODES = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP = {"e4m3": (1.75, 8), "e5m2": (1.75, 15)}   # the largest code is 1.75 * 2^8 (2^15)


def listed():
    return [
        # a decode batch of 16 tokens through one projection of width 4096: the weights are read once, latency counts
        dict(name="product-decode", kind="product", rows=16, d=4096, out=4096, a="e4m3", dtype="bf16", bias=False),
        # a prefill of 4096 tokens through the up-projection of a model of width 4096
        dict(name="product-prefill", kind="product", rows=4096, d=4096, out=11008, a="e4m3", dtype="bf16", bias=False),
        # odd sizes, results in fp32, a bias, gradients' codes on one side
        dict(name="product-ragged", kind="product", rows=1000, d=1031, out=777, a="e5m2", dtype="fp32", bias=True),
        # a classifier's head on 197 rows: launches count
        dict(name="linear-small", kind="linear", rows=197, d=256, out=1000, dtype="fp32"),
        # 64 images x 197 tokens through a projection of width 768, fp32 as the layers around it give it
        dict(name="linear-vit", kind="linear", rows=12608, d=768, out=768, dtype="fp32"),
        # 4096 tokens through a projection of width 4096, bfloat16
        dict(name="linear-lm", kind="linear", rows=4096, d=4096, out=4096, dtype="bf16"),
        # odd sizes, fp32, a plain GELU
        dict(name="act-ragged", kind="act", rows=1000, d=1031, act="gelu", gated=False, dtype="fp32", codes=False),
        # the gated MLP of a model of width 4096 on 4096 tokens, its result in 8 bits for the next product
        dict(name="act-wide", kind="act", rows=4096, d=11008, act="silu", gated=True, dtype="bf16", codes=True),
        # sampling: 16 rows of logits, the chosen token and twenty alternatives
        dict(name="logprobs-decode", kind="logprobs", rows=16, vocab=32000, tokens=1, top=20, dtype="fp32", share=1.0, masked=0.0, train=False),
        # scoring a text under a large vocabulary, five alternatives
        dict(name="logprobs-score", kind="logprobs", rows=256, vocab=128000, tokens=1, top=5, dtype="bf16", share=1.0, masked=0.0, train=False),
        # a policy's step: gradients of log probabilities and of the entropy for 4096 positions
        dict(name="logprobs-policy", kind="logprobs", rows=4096, vocab=32000, tokens=1, top=0, dtype="bf16", share=1.0, masked=0.0, train=True),
        # four candidates a position over a vocabulary of odd size, a part of which is masked out, fp32
        dict(name="logprobs-masked", kind="logprobs", rows=614, vocab=50265, tokens=4, top=8, dtype="fp32", share=0.85, masked=0.3, train=True),
    ]


def _log(rng, lo, hi, odd=0.35):
    """A size between lo and hi, even over the logarithm; most are multiples of 8, some are anything."""
    v = int(round(lo * (hi / lo) ** rng.random()))
    return max(lo, min(hi, v if v < 16 or rng.random() < odd else v // 8 * 8))


def draw(rng):
    while True:
        kind = rng.choice(["product", "product", "linear", "act", "logprobs", "logprobs"])
        if kind == "product":
            c = dict(kind=kind, rows=_log(rng, 1, 8192), d=_log(rng, 64, 8192), out=_log(rng, 64, 11008), a=rng.choice(["e4m3", "e4m3", "e5m2"]),
                     dtype=rng.choice(["bf16", "bf16", "fp32"]), bias=rng.random() < 0.3)
            if c["rows"] * c["d"] * c["out"] <= 4096 * 4096 * 11008:
                return c
        elif kind == "linear":
            c = dict(kind=kind, rows=_log(rng, 16, 16384), d=_log(rng, 64, 4096), out=_log(rng, 64, 4096), dtype=rng.choice(["bf16", "fp32"]))
            if c["rows"] * c["d"] * c["out"] <= 4096 * 4096 * 4096:
                return c
        elif kind == "act":
            c = dict(kind=kind, rows=_log(rng, 1, 16384), d=_log(rng, 32, 11008), act=rng.choice(["gelu", "silu"]), gated=rng.random() < 0.5, dtype=rng.choice(["bf16", "fp32"]))
            c["codes"] = c["dtype"] == "bf16" and rng.random() < 0.5
            if c["rows"] * c["d"] <= 4096 * 11008:
                return c
        else:
            c = dict(kind=kind, rows=_log(rng, 1, 4096), vocab=_log(rng, 100, 128000), tokens=rng.choice([1, 1, 4, 7]), top=rng.choice([0, 1, 5, 20, 32]),
                     dtype=rng.choice(["bf16", "fp32"]), share=rng.choice([1.0, 0.85]), masked=rng.choice([0.0, 0.0, 0.3]), train=rng.random() < 0.4)
            if c["rows"] * c["vocab"] <= 4096 * 32000:
                return c


# ---- inputs ----------------------------------------------------------------------------------------
def _outliers(g, x):
    """A few columns far larger than the others, as hidden states of a trained model have them."""
    d = x.shape[1]
    x[:, torch.randperm(d, generator=g, device="cuda")[:max(1, round(0.005 * d))]] *= 20.0
    return x


def _pow2(e):
    """2^e in fp32 for whole numbers from -126 to 127, by its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _blocks(x, fmt, square=False):
    """(codes as fp32, padded to whole blocks; exponents per row and block) of an fp32 matrix."""
    rows, d = x.shape
    kb, rb = -(-d // BLOCK), -(-rows // BLOCK)
    wide = torch.zeros(rb * BLOCK if square else rows, kb * BLOCK, device=x.device)
    wide[:rows, :d] = x
    a = wide.view(-1, BLOCK if square else 1, kb, BLOCK).abs().amax((1, 3))
    m, e = torch.frexp(a)
    one, up = TOP[fmt]
    e = torch.where(a > 0, e - 1 - up + (2.0 * m > one).to(e.dtype), torch.zeros_like(e))
    if square:
        e = e.repeat_interleave(BLOCK, 0)[:rows]
    wide = wide[:rows].view(rows, kb, BLOCK) * _pow2(-e)[:, :, None]
    return wide.to(CODES[fmt]).to(torch.float32).view(rows, kb * BLOCK), e


def _rounded(x, fmt, square=False):
    """The values that x has in 8 bits."""
    q, e = _blocks(x, fmt, square)
    return (q.view(x.shape[0], -1, BLOCK) * _pow2(e)[:, :, None]).view(x.shape[0], -1)[:, :x.shape[1]].contiguous()


def _stored(x, fmt, square=False):
    """Codes with the columns filled up to whole blocks, a power of two for every row and block as a byte, whole sixteens of them to a row."""
    q, e = _blocks(x, fmt, square)
    scales = torch.full((e.shape[0], -(-e.shape[1] // 16) * 16), 127, dtype=torch.uint8, device=x.device)
    scales[:, :e.shape[1]] = (e + 127).to(torch.uint8)
    return q.to(CODES[fmt]), scales.view(torch.float8_e8m0fnu)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    noise = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    st = {"case": c}
    if c["kind"] == "product":
        a, b = _outliers(g, noise(c["rows"], c["d"])), noise(c["out"], c["d"]) / math.sqrt(c["d"])
        (st["a"], st["sa"]), (st["b"], st["sb"]) = _stored(a, c["a"]), _stored(b, "e4m3", True)
        st["bias"] = noise(c["out"]) if c["bias"] else None
    elif c["kind"] == "linear":
        t = TYPES[c["dtype"]]
        st.update(x=_outliers(g, noise(c["rows"], c["d"])).to(t), w=(noise(c["out"], c["d"]) / math.sqrt(c["d"])).to(t),
                  gy=(noise(c["rows"], c["out"]) * torch.exp(noise(c["rows"], 1)) * 1e-3).to(t))
    elif c["kind"] == "act":
        t = TYPES[c["dtype"]]
        st.update(u=_outliers(g, noise(c["rows"], c["d"] * (2 if c["gated"] else 1))).to(t), g=(noise(c["rows"], c["d"]) * 1e-2).to(t))
    else:
        rows, vocab, t = c["rows"], c["vocab"], TYPES[c["dtype"]]
        logits = noise(rows, vocab) * 2.5
        if c["masked"]:
            out = torch.rand(vocab, generator=g, device="cuda") < c["masked"]
            out[0] = False
            logits[:, out] = -math.inf
        tokens = torch.randint(0, vocab, (rows, c["tokens"]), generator=g, device="cuda")
        if c["masked"]:   # a token that may not come is not asked for
            tokens = torch.where(out[tokens], torch.zeros_like(tokens), tokens)
        tokens[torch.randperm(rows, generator=g, device="cuda")[max(1, round(rows * c["share"])):]] = IGNORE
        st.update(logits=logits.to(t), tokens=tokens)
        if c["train"]:
            st.update(gp=noise(rows, c["tokens"]) / rows, gh=noise(rows) * (0.01 / rows))
    return st


# ---- plain forms -----------------------------------------------------------------------------------
def _values(codes, scales):
    rows, f = codes.shape[0], torch.float32
    s = _pow2(scales.view(torch.uint8)[:, :codes.shape[1] // BLOCK].to(torch.int32) - 127)
    return (codes.to(f).view(rows, -1, BLOCK) * s[:, :, None]).view(rows, -1)


def _plain_product(s):
    y = _values(s["a"], s["sa"]) @ _values(s["b"], s["sb"]).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return {"y": y.to(TYPES[s["case"]["dtype"]])}


def _plain_linear(s):
    f, t = torch.float32, s["x"].dtype
    x, w, gy = _rounded(s["x"].to(f), "e4m3"), _rounded(s["w"].to(f), "e4m3", True), s["gy"].to(f)
    y = x @ w.t()
    gx = _rounded(gy, "e4m3") @ w
    gw = _rounded(gy.t().contiguous(), "e4m3") @ _rounded(x.t().contiguous(), "e4m3").t()
    return {"y": y.to(t), "gx": gx.to(t), "gw": gw.to(t)}


def _act(u, act):
    """f(u) and its derivative."""
    if act == "gelu":
        phi = 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5)))
        return u * phi, phi + u * torch.exp(-0.5 * u * u) * (1.0 / math.sqrt(2.0 * math.pi))
    sig = 1.0 / (1.0 + torch.exp(-u))
    return u * sig, sig * (1.0 + u * (1.0 - sig))


def _plain_act(s):
    c, f, t, d = s["case"], torch.float32, s["u"].dtype, s["case"]["d"]
    u, g = s["u"].to(f), s["g"].to(f)
    y = _act(u[:, :d], c["act"])[0]
    if c["gated"]:
        y = y * u[:, d:]
    parts = [_rounded(p.contiguous(), "e4m3") for p in u.split(d, 1)]
    a, slope = _act(parts[0], c["act"])
    gu = torch.cat([g * slope * parts[1], g * a], 1) if c["gated"] else g * slope
    return {"y": (_rounded(y, "e4m3") if c["codes"] else y).to(t), "gu": gu.to(t)}


def _plain_logprobs(s):
    c, f = s["case"], torch.float32
    x, tokens = s["logits"].to(f), s["tokens"]
    top = x.amax(1, keepdim=True)
    lse = top + torch.log(torch.exp(x - top).sum(1, keepdim=True))
    logp = x - lse
    p = torch.exp(logp)
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    valid = tokens != IGNORE
    at = torch.where(valid, tokens, torch.zeros_like(tokens))
    out = {"logp": torch.where(valid, logp.gather(1, at), torch.zeros((), device=x.device)), "entropy": entropy}
    if c["top"]:
        # the order of the values as whole numbers, the place below it: no two alike, the lowest place first
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(torch.int64)
        keys = (order << 32) + (c["vocab"] - 1 - torch.arange(c["vocab"], device=x.device))
        best = torch.topk(keys, c["top"], dim=1, sorted=True).values
        out["top_index"] = c["vocab"] - 1 - (best & 0xFFFFFFFF)
        out["top_logp"] = logp.gather(1, out["top_index"])
    if c["train"]:
        gp = torch.where(valid, s["gp"], torch.zeros_like(s["gp"]))
        gl = -p * gp.sum(1, keepdim=True) - s["gh"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), torch.zeros_like(p))
        out["grad"] = gl.scatter_add_(1, at, gp).to(s["logits"].dtype)
    return out


# ---- the framework's entry points ------------------------------------------------------------------
def _own(s):
    from paper_2403_07339_amd import binding as imu
    c = s["case"]
    if c["kind"] == "product":
        a, b = imu.Blocks8(s["a"], s["sa"], c["d"]), imu.Blocks8(s["b"], s["sb"], c["d"])
        return {"y": imu.imunpack_block8_gemm(a, b, TYPES[c["dtype"]], bias=s["bias"])}
    if c["kind"] == "linear":
        t = s["x"].dtype
        x, _ = imu.imunpack_block8_quantize(s["x"])
        w, w_turned = imu.imunpack_block8_quantize(s["w"], square=True, turned=True)
        y = imu.imunpack_block8_gemm(x, w, t)
        gy, gy_turned = imu.imunpack_block8_quantize(s["gy"], turned=True)
        gx = imu.imunpack_block8_gemm(gy, w_turned, t)
        return {"y": y, "gx": gx, "gw": imu.imunpack_block8_gemm(gy_turned, imu.imunpack_block8_turn(x), t)}
    if c["kind"] == "act":
        y, _, kept = imu.imunpack_act8(s["u"], c["act"], gated=c["gated"], quantize=c["codes"])
        return {"y": y, "gu": imu.imunpack_act8_backward(s["g"], kept, c["act"], gated=c["gated"])}
    got = imu.imunpack_logprobs(s["logits"], s["tokens"], top=c["top"], ignore_index=IGNORE)
    out = {"logp": got.logp, "entropy": got.entropy}
    if c["top"]:
        out.update(top_index=got.top_index, top_logp=got.top_logp)
    if c["train"]:
        out["grad"] = imu.imunpack_logprobs_backward(s["logits"], s["tokens"], got, s["gp"], s["gh"], ignore_index=IGNORE)
    return out


# ---- one pass --------------------------------------------------------------------------------------
def run(state):
    if own:
        return _own(state)
    return {"product": _plain_product, "linear": _plain_linear, "act": _plain_act, "logprobs": _plain_logprobs}[state["case"]["kind"]](state)


# ---- the definition in 64 bits ---------------------------------------------------------------------
def _exact8(x, fmt, square=False):
    """Every value of a 64-bit matrix as its block's power of two and the type's few bits hold it."""
    rows, d = x.shape
    pad = torch.nn.functional.pad(x, (0, -d % BLOCK, 0, -rows % BLOCK if square else 0))
    tall = BLOCK if square else 1
    blocks = pad.reshape(pad.shape[0] // tall, tall, pad.shape[1] // BLOCK, BLOCK).transpose(1, 2)
    largest = {"e4m3": 448.0, "e5m2": 57344.0}[fmt]
    amax = blocks.abs().flatten(2).max(2).values[:, :, None, None]
    step = torch.exp2(torch.ceil(torch.log2(torch.where(amax > 0, amax / largest, torch.ones_like(amax)))))
    v = blocks / step
    bits, least = {"e4m3": (3, -6), "e5m2": (2, -14)}[fmt]
    grain = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** least))) - bits)
    v = torch.round(v / grain) * grain * step
    return v.transpose(1, 2).reshape(pad.shape)[:rows, :d]


def exact(case, seed):
    c, s, f = case, prepare(case, seed), torch.float64
    if c["kind"] == "product":
        a, b = (torch.ldexp(s[k].to(f).reshape(s[k].shape[0], -1, BLOCK), (s["s" + k].view(torch.uint8)[:, :s[k].shape[1] // BLOCK].to(f) - 127)[:, :, None]).flatten(1) for k in "ab")
        y = torch.mm(a, b.t())
        return {"y": y if s["bias"] is None else y.add_(s["bias"].to(f))}
    if c["kind"] == "linear":
        x, w, gy = _exact8(s["x"].to(f), "e4m3"), _exact8(s["w"].to(f), "e4m3", True), s["gy"].to(f)
        return {"y": torch.mm(x, w.t()), "gx": torch.mm(_exact8(gy, "e4m3"), w), "gw": torch.mm(_exact8(gy.t(), "e4m3"), _exact8(x.t(), "e4m3").t())}
    if c["kind"] == "act":
        u, g = list(s["u"].to(f).split(c["d"], 1)), s["g"].to(f)
        kept = [_exact8(p, "e4m3").requires_grad_() for p in u]
        func = (lambda v: torch.special.ndtr(v) * v) if c["act"] == "gelu" else (lambda v: v * torch.sigmoid(v))
        y = func(u[0]) * u[1] if c["gated"] else func(u[0])
        with torch.enable_grad():
            again = func(kept[0]) * kept[1] if c["gated"] else func(kept[0])
        gu = torch.cat(torch.autograd.grad(again, kept, g), 1)
        return {"y": _exact8(y, "e4m3") if c["codes"] else y, "gu": gu}
    x, tokens = s["logits"].to(f), s["tokens"]
    logp = torch.log_softmax(x, 1)
    p = logp.exp()
    entropy = torch.special.entr(p).sum(1)
    rows, place = torch.nonzero(tokens != IGNORE, as_tuple=True)
    picked = torch.zeros(tokens.shape, dtype=f, device=x.device)
    picked[rows, place] = logp[rows, tokens[rows, place]]
    out = {"logp": picked, "entropy": entropy}
    if c["top"]:
        out["top_index"] = None
        out["top_logp"] = torch.sort(logp, 1, descending=True).values[:, :c["top"]].contiguous()
    if c["train"]:
        # d logp_t = [v = t] - p_v,  dH = -p_v (log p_v + H)
        gl = p * torch.where(p > 0, logp + entropy[:, None], torch.zeros_like(p)) * -s["gh"].to(f)[:, None]
        gp = s["gp"].to(f) * (tokens != IGNORE)
        gl -= p * gp.sum(1, keepdim=True)
        gl.index_put_((rows, tokens[rows, place]), gp[rows, place], accumulate=True)
        out["grad"] = gl
    return out


# ---- what a pass cannot do without -----------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "product":
        rows, d, n = c["rows"], c["d"], c["out"]
        return {"bytes": (rows + n) * d * (1.0 + 1.0 / BLOCK) + SIZE[c["dtype"]] * rows * n, "flops": 2.0 * rows * d * n}
    if c["kind"] == "linear":    # x, w, gy in; y, gx, gw out
        rows, d, n = c["rows"], c["d"], c["out"]
        return {"bytes": 2.0 * SIZE[c["dtype"]] * (rows * d + n * d + rows * n), "flops": 6.0 * rows * d * n}
    if c["kind"] == "act":       # u in, y out, g in, gu out; what is kept is written and read
        n, wide, size = c["rows"] * c["d"], 2.0 if c["gated"] else 1.0, SIZE[c["dtype"]]
        return {"bytes": n * (2.0 * size * wide + 2.0 * size + 2.0 * wide + (1.0 if c["codes"] else 0.0)), "flops": 30.0 * n}
    n, size = c["rows"] * c["vocab"], SIZE[c["dtype"]]
    return {"bytes": n * size * (3.0 if c["train"] else 1.0) + c["rows"] * (4.0 + 12.0 * c["tokens"] + 12.0 * c["top"]), "flops": (20.0 if c["train"] else 8.0) * n}
