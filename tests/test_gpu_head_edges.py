"""GPU tests of the output head's calls at their edges, against their definitions in 64 bits.

Tolerances count roundings as test_gpu_head.py does: finfo(type).eps / 2 relative for one rounding."""
import pytest
import torch

from paper_2512_16273_b200 import tslt
from test_gpu_head import BF16, F32, gen, loss_case, loss_reference, padded, within

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
