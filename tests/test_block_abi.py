"""CPU-only checks of the feed-forward block's entry points: arguments are
refused before anything reaches the GPU."""
import ctypes

import pytest
import torch

from paper_1910_11971_amd import cci

lib = cci.raw()
P = 0x10000      # aligned, never dereferenced: validation fails first
MIS = 0x10008
F32, BF16 = cci.F32, cci.BF16
BIG = 1 << 62


def size_of(fn, *args):
    n = ctypes.c_size_t(77)
    st = fn(*args, ctypes.byref(n))
    return st, n.value


def test_exports():
    assert {"cci_layernorm", "cci_layernorm_bwd", "cci_layernorm_bwd_workspace", "cci_gated_spmm", "cci_gated_spmm_bwd",
            "cci_spmm_t", "cci_spmm_adapters", "cci_spmm_adapters_workspace"} <= set(cci.header_functions())


def norm(X=P, t=BF16, N=4, C=8, g=None, b=None, eps=1e-5, Y=P, m=None, r=None):
    return lib.cci_layernorm(X, t, N, C, g, b, eps, Y, m, r, None)


def test_layernorm_refusals():
    for kw in (dict(t=7), dict(N=-1), dict(C=0), dict(N=BIG), dict(C=BIG), dict(eps=-1.0), dict(eps=float("nan")),
               dict(X=None), dict(Y=None)):
        assert norm(**kw) == cci.EINVAL, kw
        assert lib.cci_last_error()
    for k in ("X", "g", "b", "Y", "m", "r"):
        assert norm(**{k: MIS}) == cci.EALIGN
    assert norm(N=0, X=None, Y=None) == cci.OK


def norm_bwd(dY=P, X=P, t=BF16, N=4, C=8, g=None, m=P, r=P, dX=P, dg=P, db=P, ws=P, nb=1 << 20):
    return lib.cci_layernorm_bwd(dY, X, t, N, C, g, m, r, dX, dg, db, ws, nb, None)


def test_layernorm_bwd_refusals():
    for kw in (dict(t=2), dict(N=-1), dict(C=0), dict(N=BIG), dict(dY=None), dict(X=None), dict(m=None), dict(r=None),
               dict(ws=None), dict(nb=0), dict(nb=4 * 2 * 8 - 1)):
        assert norm_bwd(**kw) == cci.EINVAL, kw
    for k in ("dY", "X", "g", "m", "r", "dX", "dg", "db", "ws"):
        assert norm_bwd(**{k: MIS}) == cci.EALIGN
    for bad in ((-1, 8), (4, 0), (BIG, BIG)):
        assert size_of(lib.cci_layernorm_bwd_workspace, *bad) == (cci.EINVAL, 77)
    assert lib.cci_layernorm_bwd_workspace(4, 8, None) == cci.EINVAL
    st, n = size_of(lib.cci_layernorm_bwd_workspace, 100000, 4096)
    assert st == cci.OK and n == 256 * 2 * 4096 * 4
    assert size_of(lib.cci_layernorm_bwd_workspace, 0, 4096) == (cci.OK, 0)


def gated(X=P, t=BF16, N=4, C=8, v=P, i=P, F=16, G=8, K=2, act=2, H=P, pre=None):
    return lib.cci_gated_spmm(X, t, N, C, v, i, F, G, K, act, H, pre, None)


def test_gated_refusals():
    for kw in (dict(t=5), dict(N=-1), dict(C=0), dict(F=12), dict(F=0), dict(G=0), dict(G=257, F=257), dict(K=0),
               dict(K=9), dict(act=5), dict(act=-1), dict(N=BIG), dict(F=1 << 60), dict(C=BIG), dict(X=None),
               dict(v=None), dict(i=None), dict(H=None)):
        assert gated(**kw) == cci.EINVAL, kw
    for k in ("X", "v", "i", "H", "pre"):
        assert gated(**{k: MIS}) == cci.EALIGN
    assert gated(N=0, X=None, v=None, i=None, H=None) == cci.OK


def gated_bwd(dH=P, pre=P, X=P, t=BF16, N=4, C=8, v=P, i=P, F=16, G=8, K=2, act=2, dp=P, dX=P, dv=P, dt=BF16):
    return lib.cci_gated_spmm_bwd(dH, pre, X, t, N, C, v, i, F, G, K, act, dp, dX, dv, dt, None)


def test_gated_bwd_refusals():
    for kw in (dict(t=5), dict(dt=5), dict(N=-1), dict(F=12), dict(K=9), dict(act=9), dict(dH=None), dict(pre=None),
               dict(dp=None), dict(v=None), dict(X=None), dict(i=None), dict(N=BIG)):
        assert gated_bwd(**kw) == cci.EINVAL, kw
    assert gated_bwd(t=F32, dt=BF16) == cci.EUNSUPPORTED
    for k in ("dH", "pre", "X", "v", "i", "dp", "dX", "dv"):
        assert gated_bwd(**{k: MIS}) == cci.EALIGN
    assert gated_bwd(N=0, dH=None, pre=None, X=None, dp=None, dv=None, dX=None, i=None) == cci.OK


def back(dY=P, t=BF16, N=4, O=16, v=P, i=P, C=8, G=8, K=2, dX=P, dt=BF16):
    return lib.cci_spmm_t(dY, t, N, O, v, i, C, G, K, dX, dt, None)


def test_spmm_t_refusals():
    for kw in (dict(t=5), dict(dt=-1), dict(N=-1), dict(O=12), dict(C=0), dict(K=0), dict(N=BIG), dict(dY=None),
               dict(v=None), dict(i=None), dict(dX=None)):
        assert back(**kw) == cci.EINVAL, kw
    assert back(t=F32, dt=BF16) == cci.EUNSUPPORTED
    for k in ("dY", "v", "i", "dX"):
        assert back(**{k: MIS}) == cci.EALIGN
    assert back(N=0, dY=None, dX=None) == cci.OK


def adapters(X=P, xt=BF16, N=4, C=8, v=P, vt=BF16, i=P, O=16, G=8, K=2, A=P, B=P, al=None, rows=P, L=2, R=4, ep=None,
             Y=P, yt=BF16, ws=P, nb=1 << 20, ad=True):
    a = cci.Adapters(A, B, al, rows, L, R)
    return lib.cci_spmm_adapters(X, xt, N, C, v, vt, i, O, G, K, ctypes.byref(a) if ad else None, ep, Y, yt, ws, nb, None)


def test_adapters_refusals():
    for kw in (dict(xt=5), dict(vt=5), dict(yt=5), dict(N=-1), dict(O=12), dict(K=9), dict(L=0), dict(L=BIG), dict(R=0),
               dict(R=1025), dict(N=BIG), dict(X=None), dict(v=None), dict(i=None), dict(Y=None), dict(A=None),
               dict(B=None), dict(rows=None), dict(ad=False), dict(ws=None), dict(nb=16)):
        assert adapters(**kw) == cci.EINVAL, kw
    for kw in (dict(vt=F32), dict(xt=F32, vt=F32, yt=BF16)):
        assert adapters(**kw) == cci.EUNSUPPORTED, kw
    for k in ("X", "v", "i", "Y", "A", "B", "al", "rows", "ws"):
        assert adapters(**{k: MIS}) == cci.EALIGN
    for k in ("scale", "bias", "residual"):
        ep = cci.Epilogue(**{k: MIS})
        assert adapters(ep=ctypes.byref(ep)) == cci.EALIGN
    assert adapters(N=0, X=None, Y=None, ws=None, A=None, B=None, rows=None) == cci.OK
    st, n = size_of(lib.cci_spmm_adapters_workspace, 33, 64, 5, 2, 4, BF16)
    assert st == cci.OK and n >= 33 * 5 * 2 + 33 * 4 * 4
    assert size_of(lib.cci_spmm_adapters_workspace, 0, 64, 5, 2, 4, BF16) == (cci.OK, 0)
    for bad in ((-1, 64, 5, 2, 4, BF16), (4, 0, 5, 2, 4, BF16), (4, 64, 0, 2, 4, BF16), (4, 64, 5, 0, 4, BF16),
                (4, 64, 5, 2, 0, BF16), (4, 64, 5, 2, 4, 9), (BIG, BIG, BIG, BIG, 4, BF16)):
        assert size_of(lib.cci_spmm_adapters_workspace, *bad) == (cci.EINVAL, 77)
    assert lib.cci_spmm_adapters_workspace(4, 64, 5, 2, 4, BF16, None) == cci.EINVAL


def test_launch_failure_without_a_device():
    if torch.cuda.is_available():
        pytest.skip("a device is there")
    assert norm() == cci.EHIP and norm_bwd() == cci.EHIP and gated() == cci.EHIP
    assert gated_bwd() == cci.EHIP and back() == cci.EHIP and adapters() == cci.EHIP


@pytest.mark.parametrize("call", [
    lambda x, v, i: cci.layernorm(x),
    lambda x, v, i: cci.layernorm_bwd(x, x, x[:, 0].contiguous(), x[:, 0].contiguous()),
    lambda x, v, i: cci.gated_spmm(x, v, i, 8),
    lambda x, v, i: cci.gated_spmm_bwd(x, x, x, v, i, 8),
    lambda x, v, i: cci.spmm_t(x, v, i, 8),
    lambda x, v, i: cci.spmm_adapters(x, v, i, 8, x, x, x),
])
def test_host_tensors_are_refused(call):
    x, v, i = torch.zeros(4, 16), torch.zeros(2, 2, 16), torch.zeros(2, 2, 16, dtype=torch.uint8)
    with pytest.raises(ValueError):
        call(x, v, i)
