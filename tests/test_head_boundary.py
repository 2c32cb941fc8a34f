"""The output head's C-ABI calls and binding without a GPU: bad arguments are refused on the host, before any launch."""
import os

import pytest
import torch


@pytest.fixture(scope="module")
def tslt():
    from paper_2512_16273_b200 import build
    build.build()
    from paper_2512_16273_b200 import tslt
    return tslt


P = 0x1000  # 16-byte aligned, never dereferenced on these paths
WS = 0x10000


def norm(t, **k):
    a = dict(x=P, r=P, w=P, dtype=1, rows=2, D=64, xs=64, rs=64, eps=1e-6, h=P, hs=64, y=P, ys=64, q=P, qs=64, scale=P)
    a.update(k)
    return t.lib().tslt_rmsnorm_quant(*[a[n] for n in ("x", "r", "w", "dtype", "rows", "D", "xs", "rs", "eps", "h", "hs", "y", "ys", "q",
                                                       "qs", "scale")], None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=P + 8), dict(xs=63), dict(xs=68), dict(r=P + 2), dict(rs=60), dict(w=P + 4), dict(h=P + 8),
                                 dict(hs=72 + 4), dict(y=P + 8), dict(ys=68), dict(q=None), dict(q=P + 8), dict(qs=72), dict(scale=None),
                                 dict(rows=-1), dict(D=0), dict(eps=-1.0), dict(eps=float("nan"))])
def test_norm_refuses(tslt, bad):
    assert norm(tslt, **bad) == tslt.ERR_INVALID_ARG


def test_norm_limits(tslt):
    assert norm(tslt, dtype=7) == tslt.ERR_UNSUPPORTED
    assert norm(tslt, D=16385, xs=16392, rs=16392, hs=16392, ys=16392, qs=16400) == tslt.ERR_UNSUPPORTED
    assert norm(tslt, rows=0, x=None, q=None) == tslt.OK
    q = tslt.lib().tslt_quantize_rows
    assert q(P, 1, 2, 64, 60, P, 64, P, None) == tslt.ERR_INVALID_ARG and q(P, 3, 2, 64, 64, P, 64, P, None) == tslt.ERR_UNSUPPORTED
    assert q(None, 1, 0, 64, 64, None, 64, None, None) == tslt.OK


def head(t, **k):
    a = dict(q=P, qs=P, qst=64, w=P, ws=P, wst=64, rows=3, V=100, D=64, dtype=1, z=P, zst=104, wsp=WS, n=4096)
    a.update(k)
    return t.lib().tslt_head_logits(*[a[n] for n in ("q", "qs", "qst", "w", "ws", "wst", "rows", "V", "D", "dtype", "z", "zst", "wsp", "n")], None)


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=P + 1), dict(qst=48), dict(qst=72), dict(qs=None), dict(w=None), dict(w=P + 8), dict(wst=63),
                                 dict(ws=None), dict(z=None), dict(z=P + 2), dict(zst=100), dict(zst=96), dict(rows=-1), dict(V=0), dict(D=0),
                                 dict(wsp=None), dict(wsp=WS + 16)])
def test_head_refuses(tslt, bad):
    assert head(tslt, **bad) == tslt.ERR_INVALID_ARG


def test_head_limits(tslt):
    assert head(tslt, dtype=2) == tslt.ERR_UNSUPPORTED
    assert head(tslt, D=65537, qst=65552, wst=65552) == tslt.ERR_UNSUPPORTED
    assert head(tslt, n=128) == tslt.ERR_WORKSPACE
    assert head(tslt, rows=(1 << 24) + 1) == tslt.ERR_UNSUPPORTED and head(tslt, V=(1 << 24) + 1, zst=1 << 25) == tslt.ERR_UNSUPPORTED
    assert head(tslt, rows=0, q=None, z=None) == tslt.OK


def fwd(lib, **k):
    a = dict(h=P, hst=64, w=P, wst=64, t=P, rows=5, V=100, D=64, loss=P, lse=P, wsp=WS, n=1 << 40)
    a.update(k)
    return lib.lib().tslt_linear_ce(*[a[n] for n in ("h", "hst", "w", "wst", "t", "rows", "V", "D", "loss", "lse", "wsp", "n")], None)


def bwd(lib, **k):
    a = dict(h=P, hst=64, w=2 * P, wst=64, t=P, lse=P, dl=None, rows=5, V=100, D=64, dh=3 * P, dhst=64, dw=4 * P, dwst=64, wsp=WS, n=1 << 40)
    a.update(k)
    return lib.lib().tslt_linear_ce_backward(*[a[n] for n in ("h", "hst", "w", "wst", "t", "lse", "dl", "rows", "V", "D", "dh", "dhst", "dw",
                                                            "dwst", "wsp", "n")], None)


COMMON = [dict(h=None), dict(h=P + 8), dict(hst=60), dict(hst=68), dict(w=None), dict(w=P + 2), dict(wst=63), dict(wst=68), dict(t=None),
          dict(lse=None), dict(rows=-1), dict(V=0), dict(D=0), dict(wsp=None), dict(wsp=WS + 128)]


@pytest.mark.parametrize("bad", COMMON + [dict(loss=None)])
def test_loss_refuses(tslt, bad):
    assert fwd(tslt, **bad) == tslt.ERR_INVALID_ARG


@pytest.mark.parametrize("bad", COMMON + [dict(dh=None), dict(dh=P + 8), dict(dhst=60), dict(dw=None), dict(dwst=68), dict(dh=P), dict(dw=2 * P),
                                          dict(dw=3 * P), dict(dw=P)])
def test_loss_backward_refuses(tslt, bad):
    assert bwd(tslt, **bad) == tslt.ERR_INVALID_ARG


def test_loss_limits(tslt):
    for call in (fwd, bwd):
        assert call(tslt, D=16392, hst=16392, wst=16392, dhst=16392, dwst=16392) == tslt.ERR_UNSUPPORTED if call is bwd else \
            call(tslt, D=16392, hst=16392, wst=16392) == tslt.ERR_UNSUPPORTED
        assert call(tslt, rows=(1 << 20) + 1) == tslt.ERR_UNSUPPORTED and call(tslt, V=(1 << 24) + 1) == tslt.ERR_UNSUPPORTED
        assert call(tslt, n=256) == tslt.ERR_WORKSPACE
    assert fwd(tslt, rows=0, h=None, t=None) == tslt.OK
    # workspaces: aligned, growing with the rows, far below the logits' size where it matters
    f = [tslt.linear_ce_workspace_bytes(r, 128256, 4096) for r in (0, 1, 100, 8192)]
    b = [tslt.linear_ce_backward_workspace_bytes(r, 128256, 4096) for r in (0, 1, 100, 8192)]
    assert all(x % 256 == 0 for x in f + b) and f == sorted(f) and b == sorted(b) and b[-1] < 8192 * 128256
    for r in (-1, (1 << 20) + 1):
        with pytest.raises(tslt.TsltError):
            tslt.linear_ce_workspace_bytes(r, 100, 64)


def test_binding_refuses_cpu_tensors(tslt):
    x = torch.zeros(2, 64)
    b = x.bfloat16()
    t = torch.zeros(2, dtype=torch.int32)
    for call in (lambda: tslt.rmsnorm_quant(x), lambda: tslt.quantize_rows(x), lambda: tslt.head_logits(x.to(torch.int8), x[:, 0], x.to(torch.int8), x[:, 0]),
                 lambda: tslt.linear_ce(b, b, t), lambda: tslt.linear_ce_backward(b, b, t, x[:, 0]), lambda: tslt.sparsify_hidden(b, None, b, x, 4)):
        with pytest.raises(ValueError):
            call()


def test_keyword_arguments(tslt):
    """Every argument can be given by its name, the first one too."""
    x = torch.zeros(2, 64)
    with pytest.raises(ValueError, match="CUDA"):
        tslt.rmsnorm_quant(x=x, eps=1e-5)
    with pytest.raises(ValueError, match="CUDA"):
        tslt.linear_ce(weight=x, target=x, hidden=x)


def test_header_and_binding_agree_on_limits(tslt):
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "tslt.h")).read()
    assert "#define TSLT_MAX_HIDDEN %d" % tslt.MAX_HIDDEN in text and "#define TSLT_MAX_INT8_K %d" % tslt.MAX_INT8_K in text
    assert "#define TSLT_MAX_LOSS_ROWS (1 << %d)" % (tslt.MAX_LOSS_ROWS.bit_length() - 1) in text
    assert "#define TSLT_MAX_VOCAB (1 << %d)" % (tslt.MAX_VOCAB.bit_length() - 1) in text
