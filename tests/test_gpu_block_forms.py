"""The feed-forward block's products on every kernel that their sizes lead to,
against the definitions in 64 bits (test_gpu_block.py's checks and bounds)."""
import pytest
import torch

import test_gpu_block as block
from block_sizes import ADAPTERS, BACK, GATED, GATED_BWD
from gpu_common import DEV, Guarded
from test_gpu_block import BF16, F32, cci, gen, normal, packed  # noqa: F401
from test_gpu_block_accuracy import check_adapters

pytestmark = pytest.mark.gpu
DT = {"bf16": BF16, "f32": F32}
sizes = lambda rows: pytest.mark.parametrize("i,size", list(enumerate(rows)))  # noqa: E731


@sizes(GATED)
def test_gated(cci, i, size):  # noqa: F811
    block.test_gated_spmm(cci, i, size[:-1], DT[size[-1]])


@sizes(GATED_BWD)
def test_gated_bwd(cci, i, size):  # noqa: F811
    block.test_gated_spmm_bwd(cci, i, size[:-1], DT[size[-1]])


@sizes(BACK)
def test_back(cci, i, size):  # noqa: F811
    block.test_spmm_t(cci, i, size[:-1], DT[size[-1]])


@sizes(ADAPTERS)
def test_adapters(cci, i, size):  # noqa: F811
    *shape, t = size
    N, C, O, G, K, L, R = shape
    dt, g = DT[t], gen(i)
    X, A, B = normal(g, N, C, dt=dt), normal(g, L, R, C, dt=dt, std=C ** -0.5), normal(g, L, O, R, dt=dt, std=R ** -0.5)
    vals, idx, W = packed(cci, g, O, C, G, K, dt)
    rows = torch.randint(-1, L, (-(-N // 5),), generator=g, device=DEV, dtype=torch.int32).repeat_interleave(5)[:N].contiguous()
    alpha, res = 1 + normal(g, L, std=0.1), normal(g, N, O, dt=dt)
    out = Guarded((N, O), dt)
    cci.spmm_adapters(X, vals, idx, G, A, B, rows, alpha=alpha, residual=res, relu=i % 2 == 0, out=out.t)
    torch.cuda.synchronize()
    check_adapters(out.t, X, W, A, B, rows, alpha, res, i % 2 == 0, f"{size}")
    out.check("adapters")
