"""Which kernels the feed-forward block's calls run on (CPU: the library's own
choice, with stand-ins for the HIP runtime)."""
import pytest

from launch_log import kernels


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
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
