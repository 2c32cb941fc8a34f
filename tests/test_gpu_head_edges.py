"""GPU tests of the output head's calls at their edges, against their definitions in 64 bits.

Tolerances count roundings as test_gpu_head.py does: finfo(type).eps / 2 relative for one rounding."""
import math
import threading

import pytest
import torch

from paper_2512_16273_b200 import tslt
from test_gpu_head import BF16, F32, U32, UBF, gen, head_case, loss_case, loss_reference, padded, within

pytestmark = pytest.mark.gpu


# ---- dloss --------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows,V", [(40, 333), (300, 900)])
@pytest.mark.parametrize("odd", [float("nan"), float("inf"), -float("inf")])
def test_linear_ce_backward_derivatives_that_are_not_finite(rows, V, odd):
    """A dloss that is not finite shows in its row's dhidden and in dweight, and in no other row's dhidden."""
    h, w, t, dl = loss_case(rows, V, 128, 0.2, 4)
    on = t >= 0
    f = tslt.linear_ce(h, w, t)
    i = int(on.nonzero()[1, 0])
    other = on.clone()
    other[i] = False
    # all of them: the usual form, one derivative for every row
    g = tslt.linear_ce_backward(h, w, t, f["lse"], torch.full_like(dl, odd))
    assert not g["dhidden"][on].isfinite().any() and not g["dweight"].isfinite().any() and not g["dhidden"][~on].any()
    # beside zeros
    one = torch.zeros_like(dl)
    one[i] = odd
    g = tslt.linear_ce_backward(h, w, t, f["lse"], one)
    assert not g["dhidden"][i].isfinite().any() and not g["dweight"].isfinite().any()
    assert not g["dhidden"][other].any() and g["dhidden"][other].isfinite().all()
    # beside finite ones: they keep their gradients bit by bit
    dl[i] = 0.0
    want = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
    dl[i] = odd
    g = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
    assert not g["dhidden"][i].isfinite().any() and not g["dweight"].isfinite().any()
    assert torch.equal(g["dhidden"][other], want["dhidden"][other])
    # in a row that is ignored: nothing
    if bool((~on).any()):
        dl[i] = 0.0
        dl[~on] = odd
        g = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
        assert torch.equal(g["dhidden"], want["dhidden"]) and torch.equal(g["dweight"], want["dweight"])


# ---- confident rows -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("where", ["even", "first", "last"])
@pytest.mark.parametrize("rows,D", [(1, 2048), (60, 2048), (200, 8192)])
def test_linear_ce_backward_confident_rows(rows, D, where):
    """Rows whose target has probability 1 - 1e-2 ... 1 - 1e-6: G there is the small difference p - 1.  `where`: the columns that the logits'
    magnitude sits in, which decides how much the tensor cores' truncating additions lose."""
    V = 1000
    g = gen(rows + D)
    wide = torch.full((D,), 0.02, device="cuda")
    if where == "even":
        wide[:] = 1.0
    elif where == "first":
        wide[:D // 16] = 1.0
    else:
        wide[-(D // 16):] = 1.0
    w = torch.randn(V, D, device="cuda", generator=g) * wide
    w = (w / w.norm(dim=1, keepdim=True)).to(BF16)
    t = torch.randperm(V, device="cuda", generator=g)[:rows].to(torch.int32)
    h = (w[t.long()].float() * torch.linspace(22.0, 12.0, rows, device="cuda")[:, None]).to(BF16)
    dl = torch.full((rows,), 0.5, device="cuda")
    hd, wd, tt = h.double(), w.double(), t.long()[:, None]
    z = hd @ wd.T
    lse = torch.logsumexp(z, 1)
    f = tslt.linear_ce(h, w, t)
    loss = lse - z.gather(1, tt)[:, 0]
    assert float(loss.min()) < 1e-4
    # zt is the same fp32 number on both sides of zt - lse, so what is left of it is lse's own: its rounding (2^-24 relative), that of
    # log2(e) as an fp32 factor (2^-25), some 16 additions to a sum near 1 (2^-24 each) and the power's 2^-22; the other entries
    # carry their logits' error, a step of 2^-23 of the magnitudes for each of D / 16 additions and as many again within them
    E = lse.abs() * 2.0 ** -23 + 2.0 ** -19
    dz = (hd.abs() @ wd.abs().T) * (D / 8 * 2 * U32) + 2.0 ** -19
    p = torch.exp(z - lse[:, None])
    gr = p.clone()
    gr.scatter_add_(1, tt, torch.full((rows, 1), -1.0, dtype=torch.float64, device="cuda"))
    others = torch.where(gr > 0, gr * dz, torch.zeros_like(gr))
    gap = others.sum(1) + E  # error of 1 - p, and of a target's entry
    within(f["loss"], loss, gap + loss * 2 * U32, "loss")
    dg = UBF * gr.abs() + torch.where(gr > 0, gr * (dz + gap[:, None]), torch.zeros_like(gr))
    dg.scatter_add_(1, tt, gap[:, None])
    o = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
    for k, want, bound in (("dhidden", gr @ wd, (dg + (V + 64) * 2 * U32 * gr.abs()) @ wd.abs()),
                           ("dweight", gr.T @ hd, (dg + (rows + 64) * 2 * U32 * gr.abs()).T @ hd.abs())):
        within(o[k], 0.5 * want, 0.5 * bound * (1 + UBF) + UBF * 0.5 * want.abs() + 1e-38, k)


# ---- norm: weights and rows that are not finite ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,D", [(1, 100), (3, 4096), (300, 64), (300, 1000), (300, 2500), (300, 5000), (2, 16384)])
def test_rmsnorm_quant_not_finite(rows, D, dtype):
    """A NaN or an infinity in the weight gives every row a scale that is NaN; one in a row gives that row's, whatever the weight."""
    g = gen(rows + D)
    x = torch.randn(rows, D, device="cuda", generator=g).to(dtype)
    w = (1 + 0.2 * torch.randn(D, device="cuda", generator=g)).to(dtype)
    x = padded(x)
    for odd in (float("nan"), float("inf"), -float("inf")):
        for at in (0, D - 1):
            v = w.clone()
            v[at] = odd
            assert tslt.rmsnorm_quant(x, v)["scale"].isnan().all()
            y, v = x.clone(), w.clone()
            y[0, at], v[at] = odd, 0.0  # the weight hides the column
            good, bad = tslt.rmsnorm_quant(padded(x.clone()), v), tslt.rmsnorm_quant(padded(y), v)
            assert bad["scale"][0].isnan() and torch.equal(bad["scale"][1:], good["scale"][1:]) and torch.equal(bad["q"][1:], good["q"][1:])


# ---- norm: sums of squares outside fp32's range ---------------------------------------------------------------
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,D", [(1, 40), (5, 4096), (300, 100), (300, 2600), (2, 16384)])
@pytest.mark.parametrize("size", [3e38, 1e25, 1e19, 1e-18, 1e-21, 1e-30, 1e-37])
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm_quant_sums_of_squares_outside_the_range(rows, D, dtype, size, residual):
    g = gen(rows + D)
    x = ((2 * torch.rand(rows, D, device="cuda", generator=g, dtype=torch.float64) - 1) * size * (0.49 if residual else 1)).to(dtype)
    r = ((2 * torch.rand(rows, D, device="cuda", generator=g, dtype=torch.float64) - 1) * size * 0.49).to(dtype) if residual else None
    w = (0.5 + 0.4 * torch.rand(D, device="cuda", generator=g)).to(dtype)
    for eps in (0.0, 1e-6):
        h = x if r is None else (x.double() + r.double()).to(dtype)
        v = (h.double() * w.double()).to(F32).double()
        top = v.abs().amax(1)
        scale = top / 127 / torch.sqrt((h.double() ** 2).mean(1) + eps)
        xp, rp = padded(x), None if r is None else padded(r)
        o = tslt.rmsnorm_quant(xp, w, rp, eps, out={"residual": xp} if residual else None)
        # fp32 sum and roundings as elsewhere; below 2^-126 the scale itself has steps of 2^-149
        within(o["scale"], scale, scale * ((D / 2 + 8) * U32) + 2.0 ** -148, "scale")
        assert torch.equal(o["q"].double(), torch.round(127 * v / top[:, None]))


# ---- a thread's first call ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("name", ["norm", "head of 3 rows", "head of 20 rows", "head of 300 rows", "loss", "gradients"])
def test_first_call_of_a_thread(name, given):
    """A thread whose first use of the device is the call itself, with a workspace given or not."""
    h, w, t, dl = loss_case(90, 500, 64, 0.0, 3)
    q, c, s, k, _ = head_case(300, 500, 64, 1)
    f = tslt.linear_ce(h, w, t)
    ws = torch.empty(tslt.linear_ce_backward_workspace_bytes(90, 500, 64), dtype=torch.uint8, device="cuda") if given else None
    call = {"norm": lambda: tslt.rmsnorm_quant(h)["q"], "head of 3 rows": lambda: tslt.head_logits(q[:3], s[:3], c, k, ws=ws)["logits"],
            "head of 20 rows": lambda: tslt.head_logits(q[:20], s[:20], c, k, ws=ws)["logits"],
            "head of 300 rows": lambda: tslt.head_logits(q, s, c, k, ws=ws)["logits"], "loss": lambda: tslt.linear_ce(h, w, t, ws=ws)["loss"],
            "gradients": lambda: tslt.linear_ce_backward(h, w, t, f["lse"], dl, ws=ws)["dweight"]}[name]
    want = call().clone()
    got = []
    torch.cuda.synchronize()
    th = threading.Thread(target=lambda: got.append(call()))
    th.start()
    th.join()
    torch.cuda.synchronize()
    assert len(got) == 1 and torch.equal(got[0], want)


# ---- workspaces and status words ------------------------------------------------------------------------------
def test_status_word_of_a_call_is_its_own():
    """What a call reports stands in the workspace that it returned, whatever the same stream runs next."""
    q, w, s, c, _ = head_case(3, 100, 64, 1)
    h, lw, t, dl = loss_case(20, 100, 64, 0.0, 9)
    t[3] = 100
    f = tslt.linear_ce(h, lw, t)
    b = tslt.linear_ce_backward(h, lw, t, f["lse"])
    z = tslt.head_logits(q, s, w, c)
    assert len({o["workspace"].data_ptr() for o in (f, b, z)}) == 3
    assert tslt.workspace_status(f["workspace"]) == tslt.workspace_status(b["workspace"]) == tslt.STATUS_BAD_TARGET
    assert tslt.workspace_status(z["workspace"]) == 0


def test_workspaces_of_calls_in_flight_are_distinct():
    """Also when a later call needs less or as much as an earlier one."""
    h, w, t, dl = loss_case(90, 500, 64, 0.0, 3)
    f = [tslt.linear_ce(h, w, t) for _ in range(3)]
    b = [tslt.linear_ce_backward(h, w, t, f[0]["lse"], dl) for _ in range(2)]
    assert len({o["workspace"].data_ptr() for o in f + b}) == 5


def test_threads_on_one_stream():
    """Threads that call on the same stream do not hand each other's rows over: the results are those of one thread alone."""
    cases = [loss_case(90, 1500, 256, 0.1 * s, 50 + s) for s in range(4)]
    want = []
    for h, w, t, dl in cases:
        f = tslt.linear_ce(h, w, t)
        b = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
        want.append([f["loss"], f["lse"], b["dhidden"], b["dweight"]])
    torch.cuda.synchronize()
    got = [[] for _ in cases]
    start = threading.Barrier(len(cases))

    def work(i):
        h, w, t, dl = cases[i]
        start.wait()
        for _ in range(40):
            f = tslt.linear_ce(h, w, t)
            b = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
            got[i].append([f["loss"], f["lse"], b["dhidden"], b["dweight"]])
    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(cases))]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert len(a) == 40 and all(torch.equal(x, y) for o in a for x, y in zip(o, b))


# ---- empty batches ----------------------------------------------------------------------------------------------
def test_status_word_of_an_empty_batch():
    h, w, t, _ = loss_case(4, 50, 64, 0.0, 1)
    q, c, s, k, _ = head_case(4, 50, 64, 1)

    def old():
        return torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")
    for give in (lambda: None, old):
        f = tslt.linear_ce(h[:0], w, t[:0], ws=give())
        b = tslt.linear_ce_backward(h[:0], w, t[:0], f["lse"], ws=give())
        z = tslt.head_logits(q[:0], s[:0], c, k, ws=give())
        assert [tslt.workspace_status(o["workspace"]) for o in (f, b, z)] == [0, 0, 0]
        assert not b["dweight"].any()


def test_status_word_of_an_empty_batch_of_logits():
    V, k = 64, 4
    z = torch.zeros(0, V, device="cuda")
    i = torch.zeros(0, k, dtype=torch.int32, device="cuda")
    f = torch.zeros(0, device="cuda")
    d = (i, torch.zeros(0, k, device="cuda"), i[:, 0].contiguous())
    par, ndr = [-1, 0], [0, -1]
    for ws in (lambda: None, lambda: torch.full((1 << 20,), 255, dtype=torch.uint8, device="cuda")):
        for o in (tslt.sparsify(z, k, ws=ws()), tslt.sparsify_shard(z, k, ws=ws()),
                  tslt.verify(z.view(0, 2, V), *d, d[2], 1.0, 1.0, f, f, ws=ws()),
                  tslt.tree_verify(z.view(0, 2, V), par, ndr, d[2], *d, 1.0, 1.0, f, f, 2, ws=ws())):
            assert tslt.workspace_status(o["workspace"]) == 0


# ---- both status words ------------------------------------------------------------------------------------------
def test_sparsify_hidden_reports_both_status_words():
    q, c, s, k, _ = head_case(4, 500, 64, 1)
    x = torch.randn(4, 64, device="cuda").to(BF16)
    o = tslt.sparsify_hidden(x, None, c, k, 8)
    assert o["head_workspace"].data_ptr() != o["workspace"].data_ptr()
    assert tslt.workspace_status(o["head_workspace"]) == 0 and tslt.workspace_status(o["workspace"]) == 0
    o["head_workspace"][:4] = torch.tensor([4, 0, 0, 0], dtype=torch.uint8)
    assert tslt.workspace_status(o["workspace"]) == 0


# ---- buffers of the exact size ----------------------------------------------------------------------------------
def exact(t, stride):
    """The rows of t at `stride`, in a buffer that ends with the last row's last element."""
    n, d = t.shape
    buf = torch.empty((n - 1) * stride + d, dtype=t.dtype, device="cuda")
    v = buf.as_strided((n, d), (stride, 1))
    v.copy_(t)
    return v


@pytest.mark.parametrize("logits", [F32, BF16])
@pytest.mark.parametrize("rows", [1, 2, 3, 4])
@pytest.mark.parametrize("D", [1, 15, 16, 17, 33, 511, 512, 527, 1601, 4090])
def test_head_logits_rows_that_end_with_their_buffer(rows, D, logits):
    V = 1003
    q, w, s, t, want = head_case(rows, V, D, rows + D)
    st = (D + 15) // 16 * 16
    z = tslt.head_logits(exact(q, st), s, exact(w, st), t, logits)["logits"]
    within(z, want, want.abs() * (3 * U32 * 1.01 + (UBF if logits == BF16 else 0)) + 1e-40, "logits")


# ---- copies out of every tile -----------------------------------------------------------------------------------
@pytest.mark.parametrize("logits", [F32, BF16])
@pytest.mark.parametrize("rows,V", [(640, 128001), (385, 100007), (200, 64 * 1501 + 1), (161, 32 * 3001 + 3), (300, 50000)])
def test_head_logits_copies_of_every_tile(rows, V, logits):
    """Many short tiles a CTA, some of whose 32-row strips or last columns are not copied out: each copy has read its box before the next
    values go in.  Integers below 2^24 and scales of 1: the fp32 logits are exact, the bf16 ones rounded once."""
    D = 64
    g = gen(rows + V)
    q = torch.randint(-127, 128, (rows, D), device="cuda", generator=g).to(torch.int8)
    w = torch.randint(-127, 128, (V, D), device="cuda", generator=g).to(torch.int8)
    one = torch.ones(max(rows, V), device="cuda")
    want = (q.double() @ w.double().T).to(F32).to(logits)
    for _ in range(10):
        z = tslt.head_logits(q, one[:rows], w, one[:V], logits)["logits"]
        assert torch.equal(z, want)


@pytest.mark.parametrize("rows,V,D", [(60, 32001, 129), (200, 32001, 257), (200, 9001, 1025), (130, 3001, 4097), (500, 20100, 64)])
def test_linear_ce_backward_copies_of_every_tile(rows, V, D):
    h, w, t, dl = loss_case(rows, V, D, 0.1, rows + D)
    d, b = loss_reference(h, w, t, dl)
    h, w = padded(h), padded(w)
    f = tslt.linear_ce(h, w, t)
    first = None
    for _ in range(10):
        g = tslt.linear_ce_backward(h, w, t, f["lse"], dl)
        if first is None:
            first = g
            for k in ("dhidden", "dweight"):
                within(g[k], d[k], b[k], k)
        assert torch.equal(g["dhidden"], first["dhidden"]) and torch.equal(g["dweight"], first["dweight"])


# ---- the bias of the tensor cores' sums ---------------------------------------------------------------------------
def correction(D):
    """What the loss multiplies a logit by, less 1: D / 16 additions that lose 0.52 units of 2^-25 of it each."""
    return D // 16 * 0.52 / 2.0 ** 25


@pytest.mark.parametrize("where", ["even", "first", "last"])
@pytest.mark.parametrize("D", [512, 4096, 8192, 16384])
def test_linear_ce_mean_error_of_lse(D, where):
    """Sums that grow evenly: the correction leaves less than half of the bias that it is there for.  0.52 is measured; half a unit lost at
    evenly spread mantissas gives 0.72, so the rest is at most 0.2 / 0.52 of it if either holds.  Sums that stand after their first
    columns lose twice as much, sums that grow in the last nothing: the correction once more, and the same half.  lse moves by
    the mean of z under the softmax."""
    rows, V = 512, 4096
    g = gen(D)
    wide = torch.full((D,), 1.0 if where == "even" else 0.02, device="cuda")
    if where != "even":
        (wide[:D // 16] if where == "first" else wide[-(D // 16):]).fill_(1.0)
    h = (torch.randn(rows, D, device="cuda", generator=g) * wide).to(BF16)
    w = (torch.randn(V, D, device="cuda", generator=g) * (3 / math.sqrt(D) / float((wide ** 2).mean()) ** 0.5)).to(BF16)
    t = torch.randint(0, V, (rows,), device="cuda", generator=g).to(torch.int32)  # (targets, whose logits are exact, hold little)
    z = h.double() @ w.double().T
    lse = torch.logsumexp(z, 1)
    bias = correction(D) * float((torch.softmax(z, 1) * z).sum(1).mean())
    err = float((tslt.linear_ce(h, w, t)["lse"].double() - lse).mean())
    # the roundings of log2(e) (2^-25 relative) and of lse itself and the power's 2^-22, at their largest in the mean
    rest = 2.0 ** -22 + float(lse.mean()) * 2.0 ** -25 + float(lse.mean()) * 2.0 ** -24 / math.sqrt(rows) * 3
    assert abs(err) <= (0.5 if where == "even" else 1.5) * bias + rest, (err, bias)


@pytest.mark.parametrize("D", [512, 4096, 16384])
@pytest.mark.parametrize("rows", [40, 300])
def test_linear_ce_sums_that_are_exact(rows, D):
    """Hidden rows with one unit that is not zero: the tensor cores lose nothing, so lse is off by the correction and fp32's roundings."""
    V = 700
    g = gen(rows + D)
    w = torch.randint(-24, 25, (V, D), device="cuda", generator=g).to(BF16)
    h = torch.zeros(rows, D, dtype=BF16, device="cuda")
    at = torch.randint(0, D, (rows,), device="cuda", generator=g)
    h[torch.arange(rows, device="cuda"), at] = 1.0
    t = torch.randint(0, V, (rows,), device="cuda", generator=g).to(torch.int32)
    z = h.double() @ w.double().T
    lse = torch.logsumexp(z, 1)
    f = tslt.linear_ce(h, w, t)
    # the factor's own rounding to fp32 (2^-24 of a logit at most), lse's rounding, the powers and additions of the sum
    bound = z.abs().amax(1) * (correction(D) + 2 * U32) + lse.abs() * U32 + 2.0 ** -19
    within(f["lse"], lse, bound, "lse")
    within(f["loss"], lse - z.gather(1, t.long()[:, None])[:, 0], bound + (lse.abs() + z.abs().amax(1)) * U32, "loss")
