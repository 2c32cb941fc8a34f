"""The output head's sources, without a GPU: rules that no result shows."""
import os

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2512_16273_b200", "csrc")


@pytest.mark.parametrize("name", ["tslt_gemm.cuh", "tslt_head.cu", "tslt_linear_ce.cu", "tslt_norm.cu"])
def test_kernels_launched_early_load_plainly(name):
    """These kernels are launched before the one before them has ended, so what they read may be written during their own life, which
    ld.global.nc (__ldg, and Elt<T>::load of the logits' kernels) does not allow."""
    text = open(os.path.join(CSRC, name)).read()
    assert "wait_for_primary_kernel" in text
    for load in ("__ldg", ".nc", "Elt<T>::load"):
        assert load not in text, load
