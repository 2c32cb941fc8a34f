"""What the output head's calls refuse beyond single bad arguments: buffers that coincide, without a GPU (every buffer is otherwise good,
and nothing is launched)."""
import pytest


@pytest.fixture(scope="module")
def tslt():
    from paper_2512_16273_b200 import build
    build.build()
    from paper_2512_16273_b200 import tslt
    return tslt


H, W, T, LOSS, LSE, WS = (0x100000 * i for i in range(1, 7))


@pytest.mark.parametrize("loss,lse", [(LOSS, LOSS), (T, LSE), (LOSS, T)])
def test_loss_outputs_that_coincide(tslt, loss, lse):
    assert tslt.lib().tslt_linear_ce(H, 64, W, 64, T, 5, 100, 64, loss, lse, WS, 1 << 40, None) == tslt.ERR_INVALID_ARG


@pytest.mark.parametrize("x,r,xs,rs,hs", [(H, W, 64, 64, 72), (H, W, 72, 64, 64), (T, H, 64, 64, 72), (T, H, 64, 80, 64)])
def test_norm_in_place_at_another_stride(tslt, x, r, xs, rs, hs):
    """residual_out is x or residual, its rows are not."""
    assert tslt.lib().tslt_rmsnorm_quant(x, r, None, tslt.BF16, 3, 64, xs, rs, 1e-6, H, hs, None, 0, LOSS, 64, LSE, None) == tslt.ERR_INVALID_ARG
