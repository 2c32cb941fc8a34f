"""GPU tests of the output head's calls (tslt_rmsnorm_quant, tslt_quantize_rows, tslt_head_logits, tslt_linear_ce and its
backward) against their definitions in 64 bits, and of a run of them together with tslt_sparsify.

Tolerances count roundings: a rounding to a type is off by at most half a step, finfo(type).eps / 2 relative.  An fp32 sum of n
products on the tensor cores is taken to be off by at most n steps of 2^-23 of the sum of the products' magnitudes (a
truncated addition loses at most one step), which the tests compute for each element in 64 bits."""
import math

import numpy as np
import pytest
import torch

from paper_2512_16273_b200 import tslt

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
U32, UBF = 2.0 ** -24, 2.0 ** -8  # half a step, relative


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def padded(t, extra=0):
    """t [rows, n] in rows of a multiple of 16 bytes, `extra` more 16-byte steps of canary behind each row."""
    step = 16 // t.element_size()
    wide = (-(-t.shape[1] // step) + extra) * step
    buf = torch.full((t.shape[0], wide), 77, dtype=torch.int8, device="cuda") if t.dtype == torch.int8 else \
        torch.full((t.shape[0], wide), float("nan"), dtype=t.dtype, device="cuda")
    buf[:, :t.shape[1]] = t
    return buf[:, :t.shape[1]]


def within(got, want, bound, what):
    err = (got.double() - want).abs()
    ok = err <= bound
    assert bool(ok.all()), "%s: %d of %d outside; worst %.3g of its bound" % (
        what, int((~ok).sum()), ok.numel(), float((err / bound.clamp_min(1e-300)).max()))


# ---- norm --------------------------------------------------------------------------------------------------
def norm_reference(x, r, w, eps):
    h = x if r is None else (x.double() + r.double()).to(x.dtype)
    f = h.double()
    v = f if w is None else (f * w.double()).to(F32).double()  # fp32 product, as defined
    top = v.abs().amax(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((f ** 2).mean(1, keepdim=True) + eps)
    q = torch.where(top > 0, torch.round(127.0 * v / top.clamp_min(1e-300)), torch.zeros_like(v))
    return h, q, torch.where(top > 0, top * rstd / 127.0, torch.zeros_like(top))[:, 0]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,D", [(1, 1), (1, 4096), (3, 7), (5, 129), (2, 16384), (700, 1000), (301, 4097), (1, 5120), (400, 64)])
@pytest.mark.parametrize("residual", [True, False])
def test_rmsnorm_quant(dtype, rows, D, residual):
    g = gen(rows * 31 + D)
    x = torch.randn(rows, D, device="cuda", generator=g).to(dtype)
    r = (3 * torch.randn(rows, D, device="cuda", generator=g)).to(dtype) if residual else None
    w = (1 + 0.3 * torch.randn(D, device="cuda", generator=g)).to(dtype)
    if rows > 2:
        x[1] = 0
        if residual:
            r[1] = 0
        x[2] *= 1e-3
    h, q, scale = norm_reference(x, r, w, 1e-6)
    o = tslt.rmsnorm_quant(padded(x, 1), w, None if r is None else padded(r, 2), 1e-6, want_values=True)
    if residual:
        assert torch.equal(o["residual"], h)
    assert torch.equal(o["q"].double(), q)
    # the sum of D squares in fp32 (relative D U32 at most, halved by the root), and a few roundings
    within(o["scale"], scale, scale * ((D / 2 + 8) * U32), "scale")
    y = q * scale[:, None]  # the scale's error, the product and the rounding to bf16
    within(o["values"], y, y.abs() * ((D / 2 + 10) * U32 + UBF * 1.01), "values")


def test_rmsnorm_quant_leaves_padding_and_works_in_place():
    g = gen(5)
    rows, D = 9, 37
    x, r = (torch.randn(rows, D, device="cuda", generator=g).to(BF16) for _ in range(2))
    h, q, scale = norm_reference(x, r, None, 0.0)
    qb = torch.full((rows, 64), 55, dtype=torch.int8, device="cuda")
    rb = padded(r, 1)
    full = rb.as_strided((rows, 48), (48, 1))
    tail = full[:, D:].clone()
    o = tslt.rmsnorm_quant(padded(x), None, rb, 0.0, out={"q": qb[:, :D], "residual": rb})
    assert torch.equal(o["q"].double(), q) and bool((qb[:, D:] == 55).all())
    assert torch.equal(rb, h) and torch.equal(full[:, D:].isnan(), tail.isnan())


def test_rmsnorm_quant_borders_and_extremes():
    """Codes at the borders between two values (ties to even), rows of the type's largest and smallest values, NaN, infinity."""
    x = torch.zeros(7, 256, device="cuda")
    x[0, :254] = torch.arange(254, device="cuda") / 2.0  # 127 v / 127 = k / 2: every tie
    x[0, 254] = 127.0
    x[1, 0] = 1e-38
    x[1, 1] = 0.5e-38
    x[2] = torch.linspace(-3e38, 3e38, 256, device="cuda")  # overflows inside: infinities and NaN
    x[6] = torch.linspace(-3e38, 3e38, 256, device="cuda", dtype=torch.float64).float()
    x[3, 5] = float("nan")
    x[4, 5] = float("inf")
    o = tslt.quantize_rows(x)
    q = o["q"].double()
    for r in (0, 1, 6):
        v = x[r].double()
        assert torch.equal(q[r], torch.round(127 * v / v.abs().max())), r
    assert bool(torch.isnan(o["scale"][2:5]).all()) and o["scale"][5] == 0 and not q[5].any()
    n = tslt.rmsnorm_quant(x[3:6], None, None, 1e-6)
    assert bool(torch.isnan(n["scale"][:2]).all()) and n["scale"][2] == 0


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_quantize_rows(dtype):
    g = gen(8)
    x = torch.randn(333, 515, device="cuda", generator=g).to(dtype)
    o = tslt.quantize_rows(padded(x))
    top = x.double().abs().amax(1, keepdim=True)
    assert torch.equal(o["q"].double(), torch.round(127 * x.double() / top))
    within(o["scale"], top[:, 0] / 127, top[:, 0] / 127 * (2 * U32), "scale")


# ---- head --------------------------------------------------------------------------------------------------
def head_case(rows, V, D, seed):
    g = gen(seed)
    q = torch.randint(-127, 128, (rows, D), device="cuda", generator=g).to(torch.int8)
    w = torch.randint(-128, 128, (V, D), device="cuda", generator=g).to(torch.int8)
    s = torch.rand(rows, device="cuda", generator=g) * 0.1
    t = torch.rand(V, device="cuda", generator=g) * 0.01
    want = (q.double() @ w.double().T) * s.double()[:, None] * t.double()[None, :]
    return q, w, s, t, want


@pytest.mark.parametrize("logits", [F32, BF16])
@pytest.mark.parametrize("rows,V,D", [(1, 1, 1), (1, 1000, 64), (2, 4099, 77), (3, 20011, 1601), (4, 515, 4096), (4, 1003, 12000), (5, 1003, 100), (16, 128, 128), (17, 129, 100), (33, 20011, 1601), (64, 4099, 2048),
                                      (65, 4099, 2048), (100, 300, 17), (256, 33000, 512), (257, 1027, 640), (700, 5001, 333)])
def test_head_logits(rows, V, D, logits):
    q, w, s, t, want = head_case(rows, V, D, rows + V + D)
    step = 8 if logits == BF16 else 4
    wide = torch.full((rows, (V + step - 1) // step * step + step), -5.0, dtype=logits, device="cuda")
    o = tslt.head_logits(padded(q), s, padded(w, 1), t, logits, out={"logits": wide[:, :V]})
    # the integer's conversion and two products in fp32; the logit's rounding
    within(o["logits"], want, want.abs() * (3 * U32 * 1.01 + (UBF if logits == BF16 else 0)) + 1e-40, "logits")
    assert bool((wide[:, V:] == -5.0).all())
    assert tslt.workspace_status(o["workspace"]) == 0


def test_head_logits_largest_sums():
    """Codes of the largest magnitude over the longest row: the sum needs all of 31 bits."""
    D = tslt.MAX_INT8_K
    q = torch.full((2, D), -128, dtype=torch.int8, device="cuda")
    w = torch.full((130, D), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one = torch.ones(130, device="cuda")
    z = tslt.head_logits(q, one[:2], w, one, F32)["logits"]
    assert z[0, 0] == 128.0 * 128 * D and z[1, 1] == -128.0 * 127 * D


# ---- loss --------------------------------------------------------------------------------------------------
def loss_case(rows, V, D, ignored, seed):
    g = gen(seed)
    w0 = torch.randn(V, D, device="cuda", generator=g).to(BF16)
    t = torch.randint(0, V, (rows,), device="cuda", generator=g)
    h = torch.randn(rows, D, device="cuda", generator=g) + torch.rand(rows, 1, device="cuda", generator=g) * (6 / math.sqrt(D)) * w0[t].float()
    w = (w0.float() * (2 / math.sqrt(D))).to(BF16)
    t = torch.where(torch.rand(rows, device="cuda", generator=g) < ignored, -1, t).to(torch.int32)
    dl = torch.randn(rows, device="cuda", generator=g)
    return h.to(BF16), w, t, dl


def loss_reference(h, w, t, dl):
    """The definitions in 64 bits, and each output's error bound."""
    on = t >= 0
    hd = torch.where(on[:, None], h.double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    wd, D, V = w.double(), h.shape[1], w.shape[0]
    z = hd @ wd.T
    lse = torch.logsumexp(z, 1)
    tt = t.clamp_min(0).long()
    loss = lse - z.gather(1, tt[:, None])[:, 0]
    dz = float((hd.abs() @ wd.abs().T).max()) * (D + 16) * 2 * U32  # error of a logit
    p = torch.exp(z - lse[:, None])
    gr = p.clone()
    gr.scatter_add_(1, tt[:, None], torch.full((len(t), 1), -1.0, dtype=torch.float64, device="cuda"))
    wt = torch.where(on, dl.double(), torch.zeros((), dtype=torch.float64, device="cuda"))[:, None]
    gr = gr * wt
    # error of a value of exp(z - lse): the logit's, the normaliser's, and those of the fp32 exponent and its power
    dp = 2 * dz + 4 * U32 * (float(z.abs().max()) + float(lse.abs().max())) * 1.5 + 2.0 ** -20
    dg = UBF * gr.abs() + dp * p * wt.abs()
    zero = torch.zeros((), dtype=torch.float64, device="cuda")
    d = {"loss": torch.where(on, loss, zero), "lse": torch.where(on, lse, zero), "dhidden": gr @ wd, "dweight": gr.T @ hd}
    n = len(t)
    b = {"lse": dz + dp + lse.abs() * U32, "loss": 2 * dz + dp + (lse.abs() + loss.abs()) * 2 * U32,
         "dhidden": (dg + (V + 64) * 2 * U32 * gr.abs()) @ wd.abs(), "dweight": (dg + (n + 64) * 2 * U32 * gr.abs()).T @ hd.abs()}
    for k in ("dhidden", "dweight"):
        b[k] = b[k] * (1 + UBF) + UBF * d[k].abs() + 1e-38
    return d, b


LOSS_SHAPES = [(1, 1, 1, 0.0), (1, 300, 64, 0.0), (5, 257, 100, 0.0), (77, 1001, 333, 0.3), (128, 4096, 256, 0.0), (129, 2000, 128, 0.5),
               (200, 5003, 72, 0.1), (500, 3001, 520, 0.2), (1100, 700, 130, 0.9)]


@pytest.mark.parametrize("rows,V,D,ignored", LOSS_SHAPES)
def test_linear_ce(rows, V, D, ignored):
    h, w, t, dl = loss_case(rows, V, D, ignored, rows + V)
    d, b = loss_reference(h, w, t, dl)
    hp = padded(h, 1)
    hp[t < 0] = float("nan")  # padding may hold anything
    f = tslt.linear_ce(hp, padded(w, 1), t)
    for k in ("loss", "lse"):
        within(f[k], d[k], torch.where(t >= 0, b[k], torch.zeros_like(b[k])), k)
    assert tslt.workspace_status(f["workspace"]) == 0


@pytest.mark.parametrize("rows,V,D,ignored", LOSS_SHAPES)
def test_linear_ce_backward(rows, V, D, ignored):
    h, w, t, dl = loss_case(rows, V, D, ignored, rows + V)
    d, b = loss_reference(h, w, t, dl)
    hp = padded(h, 1)
    hp[t < 0] = float("nan")
    wp = padded(w, 1)
    f = tslt.linear_ce(hp, wp, t)
    wide = torch.full((V, (D + 7) // 8 * 8 + 8), 7.0, dtype=BF16, device="cuda")
    g = tslt.linear_ce_backward(hp, wp, t, f["lse"], dl, out={"dweight": wide[:, :D]})
    for k in ("dhidden", "dweight"):
        within(g[k], d[k], b[k], k)
    assert not g["dhidden"][t < 0].any() and bool((wide[:, D:] == 7.0).all())
    assert tslt.workspace_status(g["workspace"]) == 0
    again = tslt.linear_ce_backward(hp, wp, t, f["lse"], dl)
    assert torch.equal(again["dhidden"], g["dhidden"]) and torch.equal(again["dweight"], g["dweight"])
