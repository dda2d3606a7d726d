"""CPU-only checks of the workspaces that the feed-forward block's calls ask for."""
import pytest
import torch

from paper_1910_11971_amd import cci
from launch_log import kernels
from test_block_abi import norm_bwd, size_of


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


@pytest.mark.parametrize("y", [cci.F32, cci.BF16])
def test_adapters_take_rows_in_slices(y, tmp_path):
    """The product's fp32 copy stays within 1 GiB, whatever the rows; each slice goes through the same launches."""
    def size(N, C, O, R):
        st, n = size_of(cci.raw().cci_spmm_adapters_workspace, N, C, O, 8, R, y)
        assert st == cci.OK
        return n

    for C, O, R in ((4096, 4096, 16), (64, 8192, 1024), (8, 8, 4)):
        rows = (1 << 28) // O // 256 * 256
        parts = 16 * 16384 * R * 4 + rows * R * 4  # column ranges of small slices, one of large ones
        for N in (1, 64, 65, rows - 1, rows, rows + 1, 3 * rows + 70, 1 << 27):
            assert size(N, C, O, R) <= (1 << 30) + parts and size(N, C, O, R) >= min(N, rows) * O * 4
    assert size(300, 8, 1 << 20, 4) >= 256 << 22
    one, two = kernels([dict(kind="adapters", N=N, C=8, O=1 << 20, G=8, K=2, L=3, R=4, dtype="bf16") for N in (256, 300)], str(tmp_path))
    names = [k.split("<")[0] for k, _, _ in two]
    assert names.count("shrink_kernel") == 2 and len([n for n in names if n.startswith("expand")]) == 2
    assert len(one) == 3 and len(two) == 6
