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
@pytest.mark.parametrize("rows,D", [(1, 1), (1, 4096), (3, 7), (5, 129), (2, 16384), (700, 1000), (301, 4097), (1, 5120), (400, 64),
                                    (299, 257), (1001, 511), (297, 1024), (303, 8)])
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
                                      (65, 4099, 2048), (100, 300, 17), (129, 5003, 257), (160, 1001, 300), (161, 1001, 300), (256, 33000, 512), (257, 1027, 640), (700, 5001, 333)])
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


@pytest.mark.parametrize("rows,V,D,ignored", LOSS_SHAPES + [(77, 32001, 1000, 0.1), (60, 225, 64, 0.0), (300, 24700, 200, 0.4)])
def test_linear_ce_reads_nothing_it_has_not_written(rows, V, D, ignored):
    """Workspaces full of NaN: the outputs are the same."""
    h, w, t, dl = loss_case(rows, V, D, ignored, rows + V)
    d, b = loss_reference(h, w, t, dl)

    h, w = padded(h), padded(w)

    def poison(n):
        return torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    f = tslt.linear_ce(h, w, t, ws=poison(tslt.linear_ce_workspace_bytes(rows, V, D)))
    g = tslt.linear_ce_backward(h, w, t, f["lse"], dl, ws=poison(tslt.linear_ce_backward_workspace_bytes(rows, V, D)))
    for k, o in (("loss", f), ("lse", f), ("dhidden", g), ("dweight", g)):
        within(o[k], d[k], torch.where(t >= 0, b[k], torch.zeros_like(b[k])) if o is f else b[k], k)


def test_linear_ce_several_pieces():
    """Rows and vocabulary at which the backward cuts the vocabulary in pieces, and dH's sum in cuts."""
    rows, V, D = 3000, 70000, 136
    assert tslt.linear_ce_backward_workspace_bytes(rows, V, D) < rows * V * 2  # less than the logits in 16 bits
    h, w, t, dl = loss_case(rows, V, D, 0.2, 3)
    d, b = loss_reference(h, w, t, dl)
    f = tslt.linear_ce(h, w, t)
    ws = torch.full((tslt.linear_ce_backward_workspace_bytes(rows, V, D),), 255, dtype=torch.uint8, device="cuda")
    g = tslt.linear_ce_backward(h, w, t, f["lse"], dl, ws=ws)
    for k, o in (("loss", f), ("lse", f)):
        within(o[k], d[k], torch.where(t >= 0, b[k], torch.zeros_like(b[k])), k)
    for k in ("dhidden", "dweight"):
        within(g[k], d[k], b[k], k)


@pytest.mark.parametrize("rows", [1, 300])
def test_linear_ce_no_row_counts(rows):
    V, D = 777, 96
    h = torch.full((rows, D), float("nan"), device="cuda", dtype=BF16)
    w = torch.randn(V, D, device="cuda").to(BF16)
    t = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    f = tslt.linear_ce(h, w, t)
    g = tslt.linear_ce_backward(h, w, t, f["lse"])
    assert not f["loss"].any() and not f["lse"].any() and not g["dhidden"].any() and not g["dweight"].any()
    assert g["dweight"].isfinite().all() and g["dhidden"].isfinite().all()


def test_empty_batches():
    w = torch.randn(50, 64, device="cuda").to(BF16)
    h, t = w[:0], torch.zeros(0, dtype=torch.int32, device="cuda")
    f = tslt.linear_ce(h, w, t)
    out = {"dweight": torch.full((50, 64), 3.0, dtype=BF16, device="cuda")}
    g = tslt.linear_ce_backward(h, w, t, f["lse"], out=out)
    assert f["loss"].shape == (0,) and g["dhidden"].shape == (0, 64) and not g["dweight"].any()
    n = tslt.rmsnorm_quant(h, w[0], h)
    assert n["q"].shape == (0, 64)
    c = tslt.quantize_rows(w)
    assert tslt.head_logits(n["q"], n["scale"], c["q"], c["scale"])["logits"].shape == (0, 50)


def test_targets_behind_the_vocabulary_are_ignored_and_reported():
    h, w, t, dl = loss_case(20, 100, 64, 0.0, 9)
    bad = t.clone()
    bad[3] = 100
    bad[7] = 2 ** 31 - 1
    f = tslt.linear_ce(h, w, bad)
    assert tslt.workspace_status(f["workspace"]) == tslt.STATUS_BAD_TARGET
    ok = torch.where(bad == t, t, -1)
    assert torch.equal(f["loss"], tslt.linear_ce(h, w, ok)["loss"]) and f["loss"][3] == 0
    g = tslt.linear_ce_backward(h, w, bad, f["lse"], dl)
    assert tslt.workspace_status(g["workspace"]) == tslt.STATUS_BAD_TARGET
    want = tslt.linear_ce_backward(h, w, ok, f["lse"], dl)
    assert torch.equal(g["dhidden"], want["dhidden"]) and torch.equal(g["dweight"], want["dweight"])
    assert tslt.workspace_status(want["workspace"]) == 0  # cleared by the next call


def test_linear_ce_not_finite():
    """A NaN or an infinity in a row that counts shows in that row's outputs and in no other row's."""
    h, w, t, _ = loss_case(40, 333, 128, 0.0, 4)
    good = tslt.linear_ce(h, w, t)
    h[5, 3] = float("nan")
    h[9, 0] = float("inf")
    f = tslt.linear_ce(h, w, t)
    rest = torch.ones(40, dtype=torch.bool, device="cuda")
    rest[[5, 9]] = False
    assert not f["loss"][5].isfinite() and not f["loss"][9].isfinite()
    assert torch.equal(f["loss"][rest], good["loss"][rest]) and torch.equal(f["lse"][rest], good["lse"][rest])
    g = tslt.linear_ce_backward(h, w, t, f["lse"])
    assert g["dhidden"][rest].isfinite().all() and not g["dhidden"][5].isfinite().any()


def test_linear_ce_equal_weights_are_a_common_factor():
    """The largest weight is taken out of the 16-bit gradients of the logits: equal weights scale the gradients exactly."""
    h, w, t, _ = loss_case(150, 999, 256, 0.3, 6)
    f = tslt.linear_ce(h, w, t)
    one = tslt.linear_ce_backward(h, w, t, f["lse"])
    third = tslt.linear_ce_backward(h, w, t, f["lse"], torch.full((150,), 0.25, device="cuda"))
    for k in ("dhidden", "dweight"):
        assert torch.equal(one[k] * 0.25, third[k])


def test_linear_ce_gradient_against_differences():
    """Directional differences of the 64-bit loss against the kernels' gradients."""
    rows, V, D = 60, 500, 96
    h, w, t, dl = loss_case(rows, V, D, 0.2, 12)
    f = tslt.linear_ce(h, w, t)
    g = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
    _, b = loss_reference(h, w, t, dl)
    on = t >= 0

    def total(hd, wd):
        z = hd[on] @ wd.T
        loss = torch.logsumexp(z, 1) - z.gather(1, t[on].long()[:, None])[:, 0]
        return float((loss * dl[on].double()).sum())
    r = gen(1)
    step = 1e-5
    for k, i in (("dhidden", 0), ("dweight", 1)):
        for _ in range(3):
            x = [h.double(), w.double()]
            e = torch.randn(x[i].shape, device="cuda", generator=r, dtype=torch.float64)
            lo, hi = list(x), list(x)
            lo[i], hi[i] = x[i] - step * e, x[i] + step * e
            diff = (total(*hi) - total(*lo)) / (2 * step)
            got = float((g[k].double() * e).sum())
            # each element's bound, and the difference quotient's own error (step^2 of a smooth function, and cancellation)
            assert abs(got - diff) <= float((b[k] * e.abs()).sum()) + 1e-6 * (1 + abs(diff))


# ---- large offsets, graphs, streams, the run together --------------------------------------------------------
def test_weights_of_more_than_2_31_elements():
    V, D = 540000, 4096
    g = gen(2)
    w = torch.randint(-127, 128, (V, D), device="cuda", generator=g, dtype=torch.int8)
    t = torch.rand(V, device="cuda", generator=g)
    for rows in (2, 20, 140):
        q = torch.randint(-127, 128, (rows, D), device="cuda", generator=g, dtype=torch.int8)
        s = torch.rand(rows, device="cuda", generator=g)
        z = tslt.head_logits(q, s, w, t, F32)["logits"]
        for v in (0, 1000, 524287, 524288, V - 1000):
            want = (q.double() @ w[v:v + 1000].double().T) * s.double()[:, None] * t[v:v + 1000].double()[None, :]
            within(z[:, v:v + 1000], want, want.abs() * (3 * U32 * 1.01) + 1e-40, "logits")
    del w, z
    V, D, rows = 140000, 16384, 20
    w = (torch.randn(V, D, device="cuda", generator=g) * 0.01).to(BF16)
    h = torch.randn(rows, D, device="cuda", generator=g).to(BF16)
    t = torch.randint(V - 2000, V, (rows,), device="cuda", generator=g).to(torch.int32)
    f = tslt.linear_ce(h, w, t)
    z = torch.cat([h.double() @ w[v:v + 20000].double().T for v in range(0, V, 20000)], 1)
    lse = torch.logsumexp(z, 1)
    # as loss_reference's bounds, with the logits' own magnitudes
    dz = max(float((h.abs().double() @ w[v:v + 20000].abs().double().T).max()) for v in range(0, V, 20000)) * (D + 16) * 2 * U32
    within(f["lse"], lse, 3 * dz + 2.0 ** -20 + lse.abs() * 4 * U32, "lse")
    b = tslt.linear_ce_backward(h, w, t, f["lse"])
    gr = torch.exp(z - lse[:, None])
    gr[torch.arange(rows, device="cuda"), t.long()] -= 1
    for v in (0, 131071, V - 2000):
        want, mag = gr[:, v:v + 2000].T @ h.double(), gr[:, v:v + 2000].abs().T @ h.double().abs()
        within(b["dweight"][v:v + 2000], want, mag * (UBF + 4 * dz + 2.0 ** -18) * 1.01 + UBF * want.abs() + 1e-30, "dweight")


def test_two_captured_graphs_do_not_share_a_workspace():
    cases = [loss_case(90, 1500, 256, 0.2, s) for s in (21, 22)]
    want = []
    for h, w, t, dl in cases:
        f = tslt.linear_ce(h, w, t)
        g = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
        want.append((f["loss"].clone(), g["dhidden"].clone(), g["dweight"].clone()))
    torch.cuda.synchronize()
    graphs, outs = [], []
    for h, w, t, dl in cases:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            f = tslt.linear_ce(h, w, t)
            g = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
        graphs.append(gr)
        outs.append((f["loss"], g["dhidden"], g["dweight"]))
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(10):
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    for o, x in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(o, x))
    # new inputs in the captured buffers
    h, w, t, dl = cases[0]
    h2, w2, t2, dl2 = loss_case(90, 1500, 256, 0.5, 23)
    f = tslt.linear_ce(h2, w2, t2)
    g = tslt.linear_ce_backward(h2, w2, t2, f["lse"], dl2)
    for a, b in ((h, h2), (w, w2), (t, t2), (dl, dl2)):
        a.copy_(b)
    graphs[0].replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[0], (f["loss"], g["dhidden"], g["dweight"])))


def test_calls_on_two_streams_at_once():
    q, w, s, t, _ = head_case(200, 30000, 512, 31)
    h, lw, lt, _ = loss_case(200, 3000, 512, 0.1, 32)
    z = tslt.head_logits(q, s, w, t)["logits"].clone()
    loss = tslt.linear_ce(h, lw, lt)["loss"].clone()
    torch.cuda.synchronize()
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    got = []
    for _ in range(8):
        with torch.cuda.stream(a):
            got.append((tslt.head_logits(q, s, w, t)["logits"], z))
            got.append((tslt.linear_ce(h, lw, lt)["loss"], loss))
        with torch.cuda.stream(b):
            got.append((tslt.linear_ce(h, lw, lt)["loss"], loss))
            got.append((tslt.head_logits(q, s, w, t)["logits"], z))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in got)


@pytest.mark.parametrize("logits", [F32, BF16])
@pytest.mark.parametrize("B,gamma", [(1, 1), (1, 4), (7, 3), (40, 5)])
def test_from_hidden_states_to_drafts_and_verification(B, gamma, logits):
    """norm -> head -> sparsify on the draft's side, norm -> head -> verify on the target's, as they are used together."""
    import oracle
    from paper_2512_16273_b200 import synth
    from parity_utils import compare_sparsify, compare_verify, verify_inputs
    V, D, k, T = 3001, 320, 32, 0.9
    g = gen(B * 10 + gamma)
    w = tslt.quantize_rows((torch.randn(V, D, device="cuda", generator=g) * (3 / math.sqrt(D))).to(BF16))
    nw = (1 + 0.1 * torch.randn(D, device="cuda", generator=g)).to(BF16)
    x, r = (torch.randn(B, gamma, D, device="cuda", generator=g).to(BF16) for _ in range(2))
    ud = synth.uniforms((B * gamma, 1), 0, synth.TID_U_DRAFT)
    s = tslt.sparsify_hidden(x, nw, w["q"], w["scale"], k, 1.0, T, ud.cuda(), residual=r, logits_dtype=logits)
    h, q, scale = norm_reference(x.reshape(-1, D), r.reshape(-1, D), nw, 1e-6)
    assert s["logits"].shape == (B, gamma, V) and torch.equal(s["residual"].reshape(-1, D), h)
    z = (q @ w["q"].double().T) * scale[:, None] * w["scale"].double()[None, :]
    within(s["logits"].reshape(-1, V), z, z.abs() * ((D / 2 + 12) * U32 + (UBF if logits == BF16 else 0)) * 1.01 + 1e-40, "logits")
    zq = s["logits"].reshape(-1, V).cpu()
    ref = oracle.sparsify(zq, k, 1.0, T, ud.numpy())
    compare_sparsify(s, ref, "hidden", logits=zq, uniforms=ud, T=T)
    # the target: one more row a sequence
    xt = torch.cat([x + 0.1 * torch.randn(x.shape, device="cuda", generator=g).to(BF16), x[:, :1]], 1)
    n = tslt.rmsnorm_quant(xt, nw, torch.cat([r, r[:, :1]], 1))
    zt = tslt.head_logits(n["q"], n["scale"], w["q"], w["scale"], logits)["logits"]
    ua = synth.uniforms((B, gamma), 0, synth.TID_U_ACCEPT)
    us = synth.uniforms((B,), 0, synth.TID_U_SAMPLE)
    tok = np.ascontiguousarray(ref["token"][:, 0].reshape(B, gamma))
    v = tslt.verify(zt, s["idx"].view(B, gamma, k), s["logit"].view(B, gamma, k), s["count"].view(B, gamma), torch.from_numpy(tok).cuda(),
                    T, T, ua.cuda(), us.cuda())
    zc = zt.cpu()
    rv = oracle.verify(zc, ref["idx"].reshape(B, gamma, k), ref["logit"].reshape(B, gamma, k), ref["count"].reshape(B, gamma), tok, T, T,
                       ua.numpy(), us.numpy())
    compare_verify(v, rv, "hidden", inputs=verify_inputs(zc, ref, B, gamma, k, tok, T, T, ua, us))


def slow_copy(dst, src, work):
    """dst = src, behind a few milliseconds of products on the same stream."""
    for _ in range(4):
        work @ work
    dst.copy_(src)


@pytest.mark.parametrize("captured", [False, True])
def test_inputs_written_on_another_stream(captured):
    """Calls whose inputs another stream writes, waited for by an event right before the call (the calls' kernels are launched
    ahead of the end of the kernel before them: an event in between has to hold them back)."""
    q, w, s, t, _ = head_case(70, 9000, 512, 41)
    h, lw, lt, dl = loss_case(70, 3000, 512, 0.1, 42)
    x = torch.randn(300, 512, device="cuda").to(BF16)

    def calls(a):
        z = tslt.head_logits(a["q"], s, w, t)["logits"]
        v = tslt.head_logits(a["q"][:3], s[:3], w, t)["logits"]
        f = tslt.linear_ce(a["h"], lw, lt)
        g = tslt.linear_ce_backward(a["h"], lw, lt, f["lse"], dl)
        n = tslt.rmsnorm_quant(a["x"])
        return [z, v, f["loss"], g["dhidden"], g["dweight"], n["q"], n["scale"]]
    want = [o.clone() for o in calls({"q": q, "h": h, "x": x})]
    buf = {"q": torch.zeros_like(q), "h": torch.zeros_like(h), "x": torch.zeros_like(x)}
    work = torch.randn(4096, 4096, device="cuda").to(BF16)
    side = torch.cuda.Stream()

    def once():
        out = []
        here = torch.cuda.current_stream()
        for k, src in (("q", q), ("h", h), ("x", x)):
            side.wait_stream(here)
            with torch.cuda.stream(side):
                slow_copy(buf[k], src, work)
            tslt.quantize_rows(x)  # a kernel of the library right before the wait
            here.wait_stream(side)
            if k == "q":
                out += [tslt.head_logits(buf[k], s, w, t)["logits"]]
            elif k == "h":
                f = tslt.linear_ce(buf[k], lw, lt)
                g = tslt.linear_ce_backward(buf[k], lw, lt, f["lse"], dl)
                out += [tslt.head_logits(buf["q"][:3], s[:3], w, t)["logits"], f["loss"], g["dhidden"], g["dweight"]]
            else:
                n = tslt.rmsnorm_quant(buf[k])
                out += [n["q"], n["scale"]]
        return out
    if captured:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            work @ work  # the product's own workspace exists before the capture
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = once()
    for _ in range(3):
        for b in buf.values():
            b.zero_()
        if captured:
            graph.replay()
        else:
            out = once()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(out, want)):
            assert torch.equal(a, b), i
