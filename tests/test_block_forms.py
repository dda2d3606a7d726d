"""Which kernels the feed-forward block's calls run on (CPU: the library's own
choice, with stand-ins for the HIP runtime)."""
import os
import random
import runpy
import shutil

import pytest

import block_sizes as sizes
import test_gpu_block as block
from launch_log import kernels

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("needs g++")
    tmp = str(tmp_path_factory.mktemp("log"))
    return lambda calls: kernels(calls, tmp)


# measured sides of the choice, far enough from its border
@pytest.mark.parametrize("C,O,G,K,on_alus,on_tiles", [
    (640, 352, 8, 2, (1, 32, 33, 64, 192), (1000,)), (128, 128, 4, 1, (1, 48, 128, 256), (257, 2000)),
    (1000, 1000, 8, 2, (1, 33, 64, 96), (192, 500)), (1024, 1024, 16, 4, (8, 33, 64), (128, 256)),
    (4096, 4096, 16, 4, (1, 8, 16), (32, 33, 64, 128)), (1024, 1024, 16, 8, (1, 16), (64, 128)),
    (1024, 256, 32, 8, (), (4, 64, 256)), (640, 352, 11, 2, (), (1, 64))])
def test_fp32_products_beside_adapters(launched, C, O, G, K, on_alus, on_tiles):
    call = lambda N: dict(kind="adapters", N=N, C=C, O=O, G=G, K=K, L=4, R=16, dtype="f32")  # noqa: E731
    for N, log in zip(on_alus, launched([call(N) for N in on_alus])):
        assert any(k.startswith("sparse_mac") for k, _, _ in log), (N, log)
    for N, log in zip(on_tiles, launched([call(N) for N in on_tiles])):
        assert any(k.startswith("tile_kernel<float, 3,") for k, _, _ in log), (N, log)


def compared() -> list[dict]:
    """The products that the GPU tests compare with their definitions."""
    out = []
    for dt in ("bf16", "f32"):
        for N, C, F, G, K in block.GATED_SIZES:
            out += [dict(kind=k, N=N, C=C, F=F, G=G, K=K, dtype=dt) for k in ("gated", "gated_bwd")]
        for N, O, C, G, K in block.BACK_SIZES:
            out += [dict(kind="back", N=N, C=C, O=O, G=G, K=K, dtype=dt, out=o) for o in (dt, "f32")]
        for N, C, O, G, K, L, R in block.ADAPTER_SIZES:
            out.append(dict(kind="adapters", N=N, C=C, O=O, G=G, K=K, L=L, R=R, dtype=dt))
    for kind, rows in (("gated", sizes.GATED), ("gated_bwd", sizes.GATED_BWD)):
        out += [dict(kind=kind, N=N, C=C, F=F, G=G, K=K, dtype=dt) for N, C, F, G, K, dt in rows]
    out += [dict(kind="back", N=N, C=C, O=O, G=G, K=K, dtype=dt) for N, O, C, G, K, dt in sizes.BACK]
    out += [dict(kind="adapters", N=N, C=C, O=O, G=G, K=K, L=L, R=R, dtype=dt) for N, C, O, G, K, L, R, dt in sizes.ADAPTERS]
    return out


def steady(kernel: str, c: dict) -> bool:
    """Whether the reduction is long enough for the kernel's loop to come round."""
    red = c["C"] if c["kind"] in ("gated", "adapters") else c["O"] if c["kind"] == "back" else 2 * c["F"]
    if kernel.startswith("wide_block_kernel"):
        return red > 8 * 64
    if kernel.startswith("wave_split_kernel"):
        wb = int(kernel.split(",")[2])
        return red >= 8 * 3 * (128 // wb)  # a third step for each of the eight waves: two or more are in flight
    return True


def test_every_kernel_of_the_ranges_is_tested(launched):
    """What thousands of drawn sizes of the performance cases' ranges run on, sizes of the GPU tests run on too, and
    with the loops of long reductions in their steady state where a drawn size has them so."""
    draw = runpy.run_path(os.path.join(ROOT, "perf", "operators.py"))
    rng = random.Random(3)
    drawn = [c for c in draw["listed"]() + [draw["draw"](rng) for _ in range(12000)] if c["kind"] not in ("norm", "norm_bwd")]
    want, have = set(), set()
    for cases, found in ((drawn, want), (compared(), have)):
        for c, log in zip(cases, launched(cases)):
            found |= {(k, steady(k, c)) for k, _, _ in log}
    missing = {(k, s) for k, s in want if (k, True) not in have and (s or (k, False) not in have)}
    assert len(want) > 100 and not missing, sorted(missing)
