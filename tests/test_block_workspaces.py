"""CPU-only checks of the workspaces that the feed-forward block's calls ask for."""
import pytest
import torch

from paper_1910_11971_amd import cci
from test_block_abi import norm_bwd


@pytest.mark.parametrize("C", [8, 16384])
def test_layernorm_bwd_without_weight_gradients_needs_none(C):
    if torch.cuda.is_available():
        pytest.skip("a device is there: made-up pointers would reach it")
    # past the checks: the launch has no device
    assert norm_bwd(C=C, dg=None, db=None, ws=None, nb=0) == cci.EHIP
    assert norm_bwd(C=C, dX=None, dg=None, db=None, ws=None, nb=0) == cci.OK  # nothing is wanted


def test_layernorm_bwd_refuses_a_missing_workspace():
    for kw in (dict(), dict(dX=None), dict(dg=None), dict(db=None), dict(C=16385, dg=None, db=None)):
        assert norm_bwd(ws=None, nb=0, **kw) == cci.EINVAL, kw
