"""The output head around libtslt's logits, as cases to be timed: the norm that quantises the hidden states, the
8-bit head product that makes the logits, and the vocabulary-wide cross entropy that trains the draft's head.

`run` gives either the plain form (elementary torch operations in 32 bits) or, where `own` is set, the calls of
paper_2512_16273_b200.tslt.  `exact` gives the same outputs from the definitions in 64 bits.
"""
import math

import torch

own = False

_BYTES = {"bf16": 2, "f32": 4}
_TYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


# ---- cases -------------------------------------------------------------------------------------------------
def _norm(rows, dim, dtype="bf16", residual=True, **more):
    return dict(more, op="norm", rows=rows, dim=dim, dtype=dtype, residual=residual)


def _head(rows, vocab, dim, logits="bf16", **more):
    return dict(more, op="head", rows=rows, vocab=vocab, dim=dim, logits=logits)


def _loss(rows, vocab, dim, ignored=0.0, grad=True, **more):
    return dict(more, op="loss", rows=rows, vocab=vocab, dim=dim, ignored=ignored, grad=grad)


def listed():
    return [
        # one draft token of one sequence: latency
        _norm(1, 4096, name="norm, one token"),
        # the gamma + 1 = 6 target rows of 32 sequences, odd width, fp32 residual stream
        _norm(192, 2561, dtype="f32", name="norm, verify rows, fp32"),
        # a prompt batch
        _norm(16384, 4096, name="norm, prompt"),
        # gamma = 4 draft positions of one sequence (the smallest workload of the benchmark), fp32 logits
        _head(4, 32000, 2048, logits="f32", name="head, 4 rows, V 32000"),
        # one draft step of 32 sequences
        _head(32, 128256, 4096, name="head, 32 rows, V 128256"),
        # ragged batch, vocabulary and width
        _head(205, 49999, 1601, name="head, 205 rows, ragged"),
        # the tree verifier's 16 x 40 target rows
        _head(640, 151936, 2048, name="head, 640 rows, V 151936"),
        # the verifier's 256 x 9 target rows of the largest workload of the benchmark
        _head(2304, 256000, 4096, name="head, 2304 rows, V 256000"),
        # scoring a held-out text: losses only
        _loss(1000, 128256, 2048, grad=False, name="loss only, 1000 rows"),
        # a small training step on a device: few tokens, odd sizes
        _loss(77, 32001, 1000, ignored=0.1, name="loss + gradients, 77 rows, ragged"),
        # an ordinary micro-batch
        _loss(2048, 32000, 2048, name="loss + gradients, 2048 rows"),
        # a large micro-batch whose prompt tokens carry no loss
        _loss(8192, 128256, 4096, ignored=0.25, name="loss + gradients, 8192 rows"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    d = _log(rng, lo, hi)
    return d if rng.random() < 0.4 else max(lo, d // 128 * 128)


def draw(rng):
    op = rng.choice(("norm", "head", "head", "loss", "loss"))
    if op == "norm":
        return _norm(_log(rng, 1, 16384), _width(rng, 512, 4096), rng.choice(("bf16", "bf16", "f32")), rng.random() < 0.7)
    if op == "head":
        return _head(_log(rng, 1, 2304), _log(rng, 8192, 256000), _width(rng, 512, 4096), rng.choice(("bf16", "bf16", "f32")))
    return _loss(_log(rng, 16, 8192), _log(rng, 8192, 128256), _width(rng, 512, 4096), rng.choice((0.0, 0.1, 0.25, 0.6)),
                 rng.random() < 0.7)


def _valid(case):
    return max(1, case["rows"] - int(case["rows"] * case["ignored"]))


def work(case):
    n, d = case["rows"], case["dim"]
    if case["op"] == "norm":
        b = _BYTES[case["dtype"]]
        return {"bytes": n * d * (b + 1 + (2 * b if case["residual"] else 0)) + d * b + 4 * n, "flops": 6 * n * d}
    v = case["vocab"]
    if case["op"] == "head":
        return {"bytes": v * d + n * d + n * v * _BYTES[case["logits"]] + 4 * (n + v), "flops": 2 * n * v * d}
    m = _valid(case)
    if case["grad"]:  # the logits, the gradient of the hidden states and that of the weight: three products
        return {"bytes": 2 * (2 * v * d + (n + m) * d) + 16 * n, "flops": 6 * m * v * d}
    return {"bytes": 2 * (v * d + m * d) + 12 * n, "flops": 2 * m * v * d}


# ---- inputs ------------------------------------------------------------------------------------------------
def _rows_of(t):
    """t [rows, n] laid out with rows of a multiple of 16 bytes, as the library asks."""
    n, step = t.shape[1], 16 // t.element_size()
    if n % step == 0:
        return t.contiguous()
    wide = torch.zeros(t.shape[0], -(-n // step) * step, dtype=t.dtype, device=t.device)
    wide[:, :n] = t
    return wide[:, :n]


def _codes(t):
    """8-bit codes and scales of the rows of t."""
    top = t.abs().amax(1, keepdim=True).clamp_min(1e-30)
    return _rows_of((t * (127.0 / top)).round_().to(torch.int8)), (top[:, 0] / 127.0).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    n, d = case["rows"], case["dim"]

    def normal(*shape):
        return torch.randn(*shape, device="cuda", generator=g)

    s = dict(case)
    if case["op"] == "norm":
        t = _TYPE[case["dtype"]]
        loud = torch.where(torch.rand(d, device="cuda", generator=g) < 0.01, 12.0, 1.0)  # a few channels are far larger
        s["x"] = _rows_of((normal(n, d) * loud).to(t))
        s["r"] = _rows_of((2.0 * normal(n, d) * loud).to(t)) if case["residual"] else None
        s["w"] = (1.0 + 0.2 * normal(d)).to(t)
        return s
    v = case["vocab"]
    if case["op"] == "head":
        s["q"], s["qs"] = _codes(normal(n, d))
        w = normal(v, d)
        w *= 2.0 / math.sqrt(d)
        s["w"], s["ws"] = _codes(w)
    else:
        w = normal(v, d).to(torch.bfloat16)
        target = torch.randint(0, v, (n,), device="cuda", generator=g)
        pull = torch.rand(n, 1, device="cuda", generator=g) * (6.0 / math.sqrt(d))  # some tokens are well predicted
        s["h"] = _rows_of((normal(n, d) + pull * w[target].float()).to(torch.bfloat16))
        w *= 2.0 / math.sqrt(d)
        s["w"] = _rows_of(w)
        m = _valid(case)
        out = torch.randperm(n, device="cuda", generator=g)[m:]
        target[out] = -1
        s["t"] = target.to(torch.int32)
        s["g"] = torch.full((n,), 1.0 / m, device="cuda")  # the mean over the tokens that count
    return s


# ---- one pass ----------------------------------------------------------------------------------------------
def run(s):
    return _own(s) if own else _plain(s)


def _own(s):
    from paper_2512_16273_b200 import tslt
    if s["op"] == "norm":
        o = tslt.rmsnorm_quant(s["x"], s["w"], s["r"], EPS, want_values=True)
        return [o["values"], o["scale"], o["residual"]] if s["r"] is not None else [o["values"], o["scale"]]
    if s["op"] == "head":
        return [tslt.head_logits(s["q"], s["qs"], s["w"], s["ws"], _TYPE[s["logits"]])["logits"]]
    f = tslt.linear_ce(s["h"], s["w"], s["t"])
    if not s["grad"]:
        return [f["loss"], f["lse"]]
    b = tslt.linear_ce_backward(s["h"], s["w"], s["t"], f["lse"], s["g"])
    return [f["loss"], f["lse"], b["dhidden"], b["dweight"]]


def _plain(s):
    if s["op"] == "norm":
        h = s["x"] if s["r"] is None else (s["x"].float() + s["r"].float()).to(s["x"].dtype)
        f = h.float()
        v = f * s["w"].float()
        top = v.abs().amax(1, keepdim=True)
        scale = top * torch.rsqrt((f * f).mean(1, keepdim=True) + EPS) / 127.0
        q = torch.where(top > 0, torch.round(v * 127.0 / top), 0.0)
        values = (q * scale).to(torch.bfloat16)
        return [values, scale[:, 0], h] if s["r"] is not None else [values, scale[:, 0]]
    if s["op"] == "head":
        z = s["q"].float() @ s["w"].float().T
        z *= s["qs"][:, None]
        z *= s["ws"][None, :]
        return [z.to(_TYPE[s["logits"]])]
    h, w = s["h"].float(), s["w"].float()
    z = h @ w.T
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    lse = (top + torch.log(total))[:, 0]
    on = s["t"] >= 0
    t = s["t"].clamp_min(0).long()[:, None]
    loss = torch.where(on, lse - z.gather(1, t)[:, 0], 0.0)
    lse = torch.where(on, lse, 0.0)
    if not s["grad"]:
        return [loss, lse]
    del z
    g = torch.where(on, s["g"], 0.0)[:, None]
    e *= g / total
    e.scatter_add_(1, t, -g)
    return [loss, lse, (e @ w).to(torch.bfloat16), (e.T @ h).to(torch.bfloat16)]


# ---- the definitions in 64 bits ----------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        x = s["x"].double()
        if s["r"] is not None:
            x = (x + s["r"].double()).to(s["x"].dtype).double()
        w = s["w"].double()
        y = x * w / torch.sqrt((x ** 2).mean(1, keepdim=True) + EPS)
        scale = y.abs().amax(1, keepdim=True) / 127
        values = torch.round(y / scale) * scale
        return [values, scale[:, 0], x] if s["r"] is not None else [values, scale[:, 0]]
    if case["op"] == "head":
        w = s["w"].double() * s["ws"].double()[:, None]
        return [torch.mm(s["q"].double() * s["qs"].double()[:, None], w.T)]
    h, w = s["h"].double(), s["w"].double()
    on = (s["t"] >= 0).nonzero()[:, 0]
    h, t = h[on], s["t"][on].long()
    z = h @ w.T
    norm = torch.logsumexp(z, 1)
    lse = torch.zeros(case["rows"], dtype=torch.float64, device="cuda")
    loss = torch.zeros_like(lse)
    lse[on] = norm
    loss[on] = norm - z[torch.arange(len(on), device="cuda"), t]
    if not case["grad"]:
        return [loss, lse]
    z.sub_(norm[:, None]).exp_()
    z[torch.arange(len(on), device="cuda"), t] -= 1
    z *= s["g"][on].double()[:, None]
    dh = torch.zeros(case["rows"], case["dim"], dtype=torch.float64, device="cuda")
    dh[on] = z @ w
    return [loss, lse, dh, z.T @ h]
