"""Feed-forward block operators on the GPU against their definitions in 64
bits: layer norm, the gated product, the transposed product and adapters.

Tolerances.  Let u = 2^-24 (half a step of fp32) and v = half a step of the
output's type (2^-24 or 2^-8).  A sum of n products taken in fp32 in any order
is off by at most n u S, S the sum of the terms' magnitudes; an output is
rounded once, by at most v |y|.  Functions of such sums pass their arguments'
errors on with their slope; the device library's exp, erf and tanh are within
a few u, for which 16 u of the factors' magnitudes are allowed.
"""
import ctypes
import math

import pytest
import torch

from gpu_common import DEV, Guarded, need_gpu

pytestmark = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
U = 2.0 ** -24
HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}
ACTS = ("silu", "gelu", "gelu_tanh", "relu", "none")
DTYPES = pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def cci():
    need_gpu()
    from paper_1910_11971_amd import cci as m
    return m


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dt=F32, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dt)


def packed(cci, g, O, C, G, K, dt):
    vals, idx = cci.pack(normal(g, O, C, std=(G / (K * C)) ** 0.5), G, K, dt)
    W = torch.zeros((O // G, G, C), dtype=F64, device=DEV)
    W.scatter_(1, idx.long(), vals.double())
    return vals, idx, W.view(O, C)


def within(got, ref, tol, what):
    assert torch.isfinite(got.double()).all(), f"{what}: not finite"
    err = (got.double() - ref).abs()
    worst = (err / tol.clamp_min(1e-300)).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: error {worst:.3g} of its bound, max {err.max().item():.3g}"


def act64(x, name):
    """act(x), act'(x) in 64 bits."""
    if name == "silu":
        s = torch.sigmoid(x)
        return x * s, s * (1 + x * (1 - s))
    if name == "gelu":
        c = torch.special.ndtr(x)
        return x * c, c + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (x + 0.044715 * x ** 3))
        return 0.5 * x * (1 + t), 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * k * (1 + 0.134145 * x * x)
    if name == "relu":
        return x.clamp_min(0), (x > 0).double()
    return x, torch.ones_like(x)


# ------------------------------------------------------------- layer norm --

NORM_SIZES = [(1, 1), (1, 7), (2, 64), (5, 100), (3, 512), (4, 513), (33, 776), (17, 1024), (9, 1025), (130, 2048),
              (6, 2049), (3, 4096), (7, 4104), (5, 8192), (3, 8193), (2, 16384), (2, 16392), (3, 40001), (1500, 72),
              (5000, 333)]


def norm_bounds(x, C):
    """Bound of the mean's error and of the relative error of rstd (a thread adds at most 48 elements, 10 levels)."""
    em = 64 * U * x.abs().mean(1, keepdim=True)
    return em, 64 * U


@DTYPES
@pytest.mark.parametrize("N,C", NORM_SIZES)
def test_layernorm(cci, N, C, dt):
    g = gen(N * 131 + C)
    X = (normal(g, N, C) * 2 + normal(g, N, 1, std=3)).to(dt)
    gamma, beta = normal(g, C) * 0.2 + 1, normal(g, C)
    for ga, be in ((gamma, beta), (None, None)):
        Y, mean, rstd = Guarded((N, C), dt), Guarded((N,), F32), Guarded((N,), F32)
        st = cci.raw().cci_layernorm(X.data_ptr(), cci._code(dt), N, C, cci._ptr(ga), cci._ptr(be), 1e-5,
                                     Y.t.data_ptr(), mean.t.data_ptr(), rstd.t.data_ptr(), None)
        assert st == cci.OK
        torch.cuda.synchronize()
        x = X.double()
        m = x.mean(1, keepdim=True)
        r = ((x - m).square().mean(1, keepdim=True) + 1e-5).rsqrt()
        em, er = norm_bounds(x, C)
        gg = (ga if ga is not None else torch.ones(C, device=DEV)).double()
        bb = (be if be is not None else torch.zeros(C, device=DEV)).double()
        within(mean.t[:, None], m, em, "mean")
        # the squares' mean moves by 2 em |d| at most, and by em^2
        within(rstd.t[:, None], r, r * (er + 4 * U) + r ** 3 * (em * (x - m).abs().mean(1, keepdim=True) + em * em), "rstd")
        xh = (x - m) * r
        ref = xh * gg + bb
        slack = (gg.abs() * (r * em * (2 + xh.abs() * (xh.abs().mean(1, keepdim=True) + 1)) + xh.abs() * (er + 8 * U))
                 + 4 * U * bb.abs())
        within(Y.t, ref, HALF[dt] * ref.abs() + slack * (1 + HALF[dt]), "Y")
        for b in (Y, mean, rstd):
            b.check("layernorm")


@DTYPES
@pytest.mark.parametrize("N,C", NORM_SIZES)
def test_layernorm_bwd(cci, N, C, dt):
    g = gen(N * 17 + C)
    X, dY = (normal(g, N, C) + normal(g, N, 1)).to(dt), normal(g, N, C, dt=dt)
    gamma = normal(g, C) * 0.2 + 1
    x, dy = X.double(), dY.double()
    mean = x.mean(1).float()
    rstd = ((x - mean.double()[:, None]).square().mean(1) + 1e-5).rsqrt().float()
    nb = ctypes.c_size_t()
    assert cci.raw().cci_layernorm_bwd_workspace(N, C, ctypes.byref(nb)) == cci.OK
    for ga, want_dx in ((gamma, True), (None, True), (gamma, False)):
        dX, dg, db = Guarded((N, C), dt), Guarded((C,), F32), Guarded((C,), F32)
        ws = Guarded((nb.value,), torch.uint8)
        st = cci.raw().cci_layernorm_bwd(dY.data_ptr(), X.data_ptr(), cci._code(dt), N, C, cci._ptr(ga),
                                         mean.data_ptr(), rstd.data_ptr(), dX.t.data_ptr() if want_dx else None,
                                         dg.t.data_ptr(), db.t.data_ptr(), ws.t.data_ptr(), nb.value, None)
        assert st == cci.OK
        torch.cuda.synchronize()
        m, r = mean.double()[:, None], rstd.double()[:, None]
        gg = (ga if ga is not None else torch.ones(C, device=DEV)).double()
        xh, q = (x - m) * r, dy * gg
        exh = 4 * U * ((x.abs() + m.abs()) * r)  # of xh in fp32
        within(db.t, dy.sum(0), N * U * dy.abs().sum(0), "dbeta")
        within(dg.t, (dy * xh).sum(0), (N + 2) * U * (dy * xh).abs().sum(0) + (dy.abs() * exh).sum(0), "dgamma")
        if want_dx:
            c1, c2 = q.mean(1, keepdim=True), (q * xh).mean(1, keepdim=True)
            ref = r * (q - c1 - xh * c2)
            e1 = 64 * U * q.abs().mean(1, keepdim=True)
            e2 = 64 * U * (q * xh).abs().mean(1, keepdim=True) + (q.abs() * exh).mean(1, keepdim=True)
            slack = r * (e1 + xh.abs() * e2 + exh * c2.abs() + 8 * U * (q.abs() + c1.abs() + (xh * c2).abs()))
            within(dX.t, ref, HALF[dt] * ref.abs() + slack * (1 + HALF[dt]), "dX")
        for b in (dX, dg, db, ws):
            b.check("layernorm_bwd")


def test_layernorm_empty_and_special(cci):
    dX, dg, db = cci.layernorm_bwd(torch.empty((0, 9), device=DEV), torch.empty((0, 9), device=DEV),
                                   torch.empty(0, device=DEV), torch.empty(0, device=DEV))
    assert dX.shape == (0, 9) and (dg == 0).all() and (db == 0).all()
    assert cci.layernorm(torch.empty((0, 9), device=DEV))[0].shape == (0, 9)
    X = torch.ones((3, 40), device=DEV)            # a row of equal values: 0 / sqrt(eps)
    X[1, 5] = float("inf")                          # touches its own row alone
    Y, mean, rstd = cci.layernorm(X, eps=1e-5)
    assert (Y[0] == 0).all() and (Y[2] == 0).all() and Y[1].isnan().all()
    # far from zero the deviations keep their digits: two values a step apart
    X = torch.full((2, 64), 4096.0, device=DEV)
    X[:, ::2] += 2.0 ** -11
    Y, mean, rstd = cci.layernorm(X, eps=0.0)
    x = X.double()
    xh = (x - x.mean(1, keepdim=True)) / x.std(1, correction=0, keepdim=True)
    assert (Y.double() - xh).abs().max() < 1e-5


def test_layernorm_bwd_against_differences(cci):
    g = gen(5)
    N, C, eps = 3, 11, 1e-5
    X, dY, gamma, beta = normal(g, N, C), normal(g, N, C), normal(g, C), normal(g, C)
    _, mean, rstd = cci.layernorm(X, gamma, beta, eps)
    got = cci.layernorm_bwd(dY, X, mean, rstd, gamma)

    def loss(x, ga, be):
        d = x - x.mean(1, keepdim=True)
        return ((d / (d.square().mean(1, keepdim=True) + eps).sqrt() * ga + be) * dY.double()).sum()

    args = [X.double(), gamma.double(), beta.double()]
    for i, grad in enumerate(got):
        num = torch.zeros_like(args[i])
        for j in range(num.numel()):
            e = torch.zeros_like(args[i]).view(-1)
            e[j] = 1e-5
            e = e.view_as(args[i])
            hi, lo = list(args), list(args)
            hi[i], lo[i] = args[i] + e, args[i] - e
            num.view(-1)[j] = (loss(*hi) - loss(*lo)) / 2e-5
        assert (grad.double() - num).abs().max() < 1e-4 * max(1.0, num.abs().max().item())


# ----------------------------------------------------------- gated product --

GATED_SIZES = [(1, 8, 8, 8, 2), (1, 64, 96, 16, 4), (3, 5, 6, 3, 2), (16, 128, 256, 16, 4), (17, 33, 40, 4, 1),
               (37, 520, 144, 16, 4), (64, 64, 64, 16, 4), (65, 72, 96, 32, 8), (130, 200, 256, 256, 3),
               (33, 96, 512, 256, 256), (129, 64, 160, 16, 16), (200, 129, 130, 2, 1), (70, 1000, 48, 8, 8),
               (3333, 264, 1736, 8, 2), (1999, 448, 3104, 32, 20), (2500, 1000, 2544, 16, 16),
               (2048, 512, 2560, 16, 4), (4100, 256, 1536, 64, 4),
               (90, 520, 512, 64, 40), (5, 1, 1, 1, 1), (2049, 136, 1032, 8, 2), (300, 256, 384, 16, 4),
               (2100, 64, 1100, 4, 2), (1024, 320, 2048, 32, 8)]


def gated_ref(X, W, F, act):
    x = X.double()
    P, S = x @ W.t(), x.abs() @ W.abs().t()
    a, _ = act64(P[:, :F], act)
    return P, S, a * P[:, F:], a


@DTYPES
@pytest.mark.parametrize("i,size", list(enumerate(GATED_SIZES)))
def test_gated_spmm(cci, i, size, dt):
    N, C, F, G, K = size
    g = gen(i)
    X = normal(g, N, C, dt=dt)
    vals, idx, W = packed(cci, g, 2 * F, C, G, K, dt)
    for act, save in ((ACTS[i % 5], True), (ACTS[(i + 1) % 5], False)):
        H, pre = Guarded((N, F), dt), Guarded((N, 2 * F), dt)
        st = cci.raw().cci_gated_spmm(X.data_ptr(), cci._code(dt), N, C, vals.data_ptr(), idx.data_ptr(), F, G, K,
                                      cci.ACTS[act], H.t.data_ptr(), pre.t.data_ptr() if save else None, None)
        assert st == cci.OK, cci.raw().cci_last_error()
        torch.cuda.synchronize()
        P, S, ref, a = gated_ref(X, W, F, act)
        e = (C + 2) * U * S
        if save:
            within(pre.t, P, HALF[dt] * P.abs() + e * (1 + HALF[dt]), "pre")
        gt, ut, eg, eu = P[:, :F], P[:, F:], e[:, :F], e[:, F:]
        slack = 1.2 * eg * (ut.abs() + eu) + a.abs() * eu + 16 * U * gt.abs() * ut.abs()
        within(H.t, ref, HALF[dt] * ref.abs() + slack * (1 + HALF[dt]), f"H {act}")
        H.check("gated H"), pre.check("gated pre")


@DTYPES
@pytest.mark.parametrize("i,size", list(enumerate(GATED_SIZES)))
def test_gated_spmm_bwd(cci, i, size, dt):
    N, C, F, G, K = size
    g = gen(100 + i)
    X, pre, dH = normal(g, N, C, dt=dt), normal(g, N, 2 * F, dt=dt, std=2), normal(g, N, F, dt=dt)
    vals, idx, W = packed(cci, g, 2 * F, C, G, K, dt)
    act = ACTS[i % 5]
    for dv_t in {dt, F32}:
        dpre, dX, dv = Guarded((N, 2 * F), dt), Guarded((N, C), dt), Guarded(vals.shape, dv_t)
        st = cci.raw().cci_gated_spmm_bwd(dH.data_ptr(), pre.data_ptr(), X.data_ptr(), cci._code(dt), N, C,
                                          vals.data_ptr(), idx.data_ptr(), F, G, K, cci.ACTS[act], dpre.t.data_ptr(),
                                          dX.t.data_ptr(), dv.t.data_ptr(), cci._code(dv_t), None)
        assert st == cci.OK, cci.raw().cci_last_error()
        torch.cuda.synchronize()
        p, dh = pre.double(), dH.double()
        gt, ut = p[:, :F], p[:, F:]
        a, da = act64(gt, act)
        ref = torch.cat((dh * ut * da, dh * a), 1)
        slack = torch.cat(((dh * ut).abs() * 32 * U * (2 + gt.abs()), dh.abs() * 16 * U * gt.abs()), 1)
        within(dpre.t, ref, HALF[dt] * ref.abs() + slack * (1 + HALF[dt]), f"dpre {act}")
        # the two products read dpre as it was returned
        d = dpre.t.double()
        check_product(dX.t, d, W, 2 * F, "dX")
        check_grad(dv.t, d, X.double(), idx, G, "dvals")
        for b in (dpre, dX, dv):
            b.check("gated_bwd")


def check_product(got, d, W, n, what):
    ref, S = d @ W, d.abs() @ W.abs()
    within(got, ref, HALF[got.dtype] * ref.abs() + (n + 2) * U * S * (1 + HALF[got.dtype]), what)


def check_grad(got, d, x, idx, G, what):
    shape = (idx.shape[0], G, idx.shape[2])
    ref = (d.t() @ x).view(shape).gather(1, idx.long())
    S = (d.abs().t() @ x.abs()).view(shape).gather(1, idx.long())
    within(got, ref, HALF[got.dtype] * ref.abs() + (d.shape[0] + 2) * U * S * (1 + HALF[got.dtype]), what)


def test_gated_bwd_parts_and_empty(cci):
    g = gen(7)
    N, C, F, G, K = 40, 72, 48, 8, 2
    X, pre, dH = normal(g, N, C, dt=BF16), normal(g, N, 2 * F, dt=BF16), normal(g, N, F, dt=BF16)
    vals, idx, _ = packed(cci, g, 2 * F, C, G, K, BF16)
    whole = cci.gated_spmm_bwd(dH, pre, X, vals, idx, G)
    some = cci.gated_spmm_bwd(dH, pre, X, vals, idx, G, need_dx=False)
    assert some[1] is None and torch.equal(whole[0], some[0]) and torch.equal(whole[2], some[2])
    some = cci.gated_spmm_bwd(dH, pre, X, vals, idx, G, need_dvals=False)
    assert some[2] is None and torch.equal(whole[1], some[1])
    e = lambda w: torch.empty((0, w), dtype=BF16, device=DEV)  # noqa: E731
    dpre, dX, dv = cci.gated_spmm_bwd(e(F), e(2 * F), e(C), vals, idx, G)
    assert dpre.shape == (0, 2 * F) and dX.shape == (0, C) and (dv == 0).all()
    assert cci.gated_spmm(e(C), vals, idx, G).shape == (0, F)
    assert cci.spmm_t(e(2 * F), vals, idx, G).shape == (0, C)


def test_gated_bwd_against_differences(cci):
    g = gen(9)
    N, C, F, G, K = 3, 5, 4, 2, 1
    X, dH = normal(g, N, C), normal(g, N, F)
    vals, idx, _ = packed(cci, g, 2 * F, C, G, K, F32)
    for act in ("silu", "gelu", "gelu_tanh", "none"):
        _, pre = cci.gated_spmm(X, vals, idx, G, act=act, save_pre=True)
        _, dX, dv = cci.gated_spmm_bwd(dH, pre, X, vals, idx, G, act=act)

        def loss(x, v):
            W = torch.zeros((2 * F // G, G, C), dtype=F64, device=DEV).scatter_(1, idx.long(), v).view(2 * F, C)
            P = x @ W.t()
            return (act64(P[:, :F], act)[0] * P[:, F:] * dH.double()).sum()

        for i, grad in enumerate((dX, dv)):
            args = [X.double(), vals.double()]
            num = torch.zeros_like(args[i])
            for j in range(num.numel()):
                e = torch.zeros(num.numel(), dtype=F64, device=DEV)
                e[j] = 1e-5
                hi, lo = list(args), list(args)
                hi[i], lo[i] = args[i] + e.view_as(num), args[i] - e.view_as(num)
                num.view(-1)[j] = (loss(*hi) - loss(*lo)) / 2e-5
            assert (grad.double() - num).abs().max() < 1e-5 * max(1.0, num.abs().max().item())


def test_gated_far_arguments(cci):
    """Preactivations far out: the activations and their slopes stay finite where their values are."""
    G = K = 1
    X = torch.tensor([[1.0], [-1.0], [0.0]], device=DEV)
    W = torch.tensor([[3e4], [1e20], [3e38], [2.0], [2.0], [2.0]], device=DEV)
    vals, idx = cci.pack(W, G, K, F32)
    for act in ACTS:
        H, pre = cci.gated_spmm(X, vals, idx, G, act=act, save_pre=True)
        a, da = act64(pre[:, :3].double().clamp(-1e12, 1e12), act)
        dpre, _, _ = cci.gated_spmm_bwd(torch.ones_like(H), pre, X, vals, idx, G, act=act)
        if act in ("relu", "none"):
            continue  # (3e38 * 2 is not finite there, nor has it to be)
        assert torch.isfinite(dpre[:, :3]).all(), act
        assert torch.allclose(dpre[:, :3].double(), 2 * X.double() * da, atol=1e-5), act


def test_non_finite_rows_stay_apart(cci):
    g = gen(11)
    N, C, F, G, K = 70, 64, 96, 8, 2
    X = normal(g, N, C, dt=BF16)
    vals, idx, _ = packed(cci, g, 2 * F, C, G, K, BF16)
    clean = cci.gated_spmm(X, vals, idx, G)
    dY = normal(g, N, 2 * F, dt=BF16)
    back = cci.spmm_t(dY, vals, idx, G)
    X[3, 7], X[40, 0] = float("nan"), float("inf")
    dY[5, 9] = float("-inf")
    H, dX = cci.gated_spmm(X, vals, idx, G), cci.spmm_t(dY, vals, idx, G)
    keep = torch.ones(N, dtype=torch.bool, device=DEV)
    keep[[3, 40]] = False
    assert torch.equal(H[keep], clean[keep]) and not torch.isfinite(H[3]).all() and not torch.isfinite(H[40]).all()
    keep = torch.arange(N, device=DEV) != 5
    assert torch.equal(dX[keep], back[keep]) and not torch.isfinite(dX[5]).all()


# ------------------------------------------------------ transposed product --

BACK_SIZES = [(1, 8, 8, 8, 2), (1, 4096, 64, 16, 4), (3, 6, 5, 3, 2), (64, 64, 64, 16, 4), (33, 96, 129, 32, 8),
              (100, 512, 200, 256, 7), (70, 256, 264, 256, 256), (2049, 72, 2050, 8, 2), (2048, 512, 2048, 16, 4),
              (300, 1040, 512, 16, 16), (3333, 1736, 3400, 8, 2), (6001, 400, 2056, 16, 9), (4096, 320, 3136, 2, 1),
              (4000, 640, 4000, 64, 64), (8192, 256, 1792, 16, 1), (257, 130, 131, 2, 1), (90, 960, 256, 64, 33),
              (40, 21, 1, 7, 3)]


@DTYPES
@pytest.mark.parametrize("i,size", list(enumerate(BACK_SIZES)))
def test_spmm_t(cci, i, size, dt):
    N, O, C, G, K = size
    g = gen(200 + i)
    dY = normal(g, N, O, dt=dt)
    vals, idx, W = packed(cci, g, O, C, G, K, dt)
    for y_t in {dt, F32}:
        out = Guarded((N, C), y_t)
        got = cci.spmm_t(dY, vals, idx, G, out_dtype=y_t, out=out.t)
        torch.cuda.synchronize()
        check_product(got, dY.double(), W, O, "dX")
        out.check("spmm_t")


# ---------------------------------------------------------------- adapters --

ADAPTER_SIZES = [(1, 8, 8, 8, 2, 1, 1), (1, 4096, 256, 16, 4, 4, 16), (32, 512, 256, 16, 4, 16, 16),
                 (64, 256, 128, 8, 2, 100, 8), (37, 96, 130, 2, 1, 3, 5), (200, 72, 200, 8, 2, 5, 64),
                 (333, 129, 48, 4, 1, 7, 33), (100, 64, 66, 3, 2, 2, 16), (1000, 320, 264, 8, 4, 9, 100),
                 (50, 1000, 256, 64, 8, 3, 4), (2, 33, 21, 7, 7, 2, 257), (150, 64, 200, 8, 2, 3, 600),
                 (70, 160, 90, 2, 1, 2, 48), (500, 544, 96, 16, 4, 70, 16), (65, 31, 65, 5, 2, 1, 1024),
                 (239, 3896, 416, 32, 8, 5, 32)]


@DTYPES
@pytest.mark.parametrize("order", ["any", "runs"])
@pytest.mark.parametrize("i,size", list(enumerate(ADAPTER_SIZES)))
def test_spmm_adapters(cci, i, size, order, dt):
    N, C, O, G, K, L, R = size
    g = gen(300 + i)
    X, A, B = normal(g, N, C, dt=dt), normal(g, L, R, C, dt=dt, std=C ** -0.5), normal(g, L, O, R, dt=dt, std=R ** -0.5)
    vals, idx, W = packed(cci, g, O, C, G, K, dt)
    rows = torch.randint(-2, L + 2, (N,), generator=g, device=DEV, dtype=torch.int32)
    if order == "runs":
        rows = rows[:-(-N // 7)].repeat_interleave(7)[:N].contiguous()
    alpha, scale, bias = normal(g, L), normal(g, O), normal(g, O)
    for y_t in {dt, F32}:
        res = normal(g, N, O, dt=y_t)
        for al, sc, bi, rs, relu in ((alpha, scale, bias, res, True), (None, None, None, None, False)):
            out = Guarded((N, O), y_t)
            got = cci.spmm_adapters(X, vals, idx, G, A, B, rows, alpha=al, scale=sc, bias=bi, residual=rs, relu=relu, out_dtype=y_t,
                                    out=out.t)
            torch.cuda.synchronize()
            x = X.double()
            acc, S = x @ W.t(), x.abs() @ W.abs().t()
            D = rs.double() if rs is not None else torch.zeros((N, O), dtype=F64, device=DEV)
            SD = torch.zeros((N, O), dtype=F64, device=DEV)  # magnitudes of the adapter's terms
            for a in range(L):
                n = (rows == a).nonzero()[:, 0]
                f = al[a].double() if al is not None else 1.0
                D[n] += f * (x[n] @ A[a].double().t()) @ B[a].double().t()
                SD[n] += abs(f) * (x[n].abs() @ A[a].double().abs().t()) @ B[a].double().abs().t()
            if sc is not None:
                acc, S = acc * sc.double() + bi.double(), S * sc.double().abs() + bi.double().abs()
            # bf16: the low part of T is rounded to 8 bits below the high part's 8: 2^-16 of each term
            eD = ((C + R + 24) * U + (2.0 ** -16 if dt == BF16 else 0.0)) * SD + 2 * U * D.abs()
            ref = acc + D
            e = (C + 6) * U * S + eD + HALF[y_t] * (D.abs() + eD) + 2 * U * (D.abs() + S)
            if relu:
                ref = ref.clamp_min(0)
            within(got, ref, HALF[y_t] * ref.abs() + e * (1 + HALF[y_t]), f"adapters {y_t}")
            out.check("adapters")


def test_adapters_without_any(cci):
    g = gen(12)
    N, C, O, G, K = 40, 64, 48, 8, 2
    X, bias = normal(g, N, C, dt=BF16), normal(g, O)
    vals, idx, _ = packed(cci, g, O, C, G, K, BF16)
    A, B = normal(g, 3, 8, C, dt=BF16), normal(g, 3, O, 8, dt=BF16)
    A[1] = float("nan")  # not read into rows without that adapter
    rows = torch.full((N,), -1, device=DEV, dtype=torch.int32)
    plain = cci.spmm(X, vals, idx, G, bias=bias)
    assert torch.equal(cci.spmm_adapters(X, vals, idx, G, A, B, rows, bias=bias), plain)
    rows[:] = torch.arange(N, device=DEV) % 3
    mixed = cci.spmm_adapters(X, vals, idx, G, A, B, rows, bias=bias)
    assert mixed[1::3].isnan().all() and torch.isfinite(mixed[0::3]).all() and torch.isfinite(mixed[2::3]).all()
    e = torch.empty((0, C), dtype=BF16, device=DEV)
    assert cci.spmm_adapters(e, vals, idx, G, A, B, rows[:0]).shape == (0, O)


# ---------------------------------------------------------- used together --

def block(cci, s, train):
    """norm -> gated product -> down projection, and back."""
    y, mean, rstd = cci.layernorm(s["x"], s["gamma"], s["beta"])
    if not train:
        h = cci.gated_spmm(y, *s["up"], 16)
        return (cci.spmm_adapters(h, *s["down"], 16, s["A"], s["B"], s["rows"], residual=s["x"]),)
    h, pre = cci.gated_spmm(y, *s["up"], 16, save_pre=True)
    out = cci.spmm(h, *s["down"], 16, residual=s["x"])
    dh = cci.spmm_t(s["dout"], *s["down"], 16)
    dv_down = cci.grad_packed(s["dout"], h, s["down"][1], 16)
    _, dy, dv_up = cci.gated_spmm_bwd(dh, pre, y, *s["up"], 16)
    dx, dg, db = cci.layernorm_bwd(dy, s["x"], mean, rstd, s["gamma"])
    return out, dx, dg, db, dv_up, dv_down


def block_state(cci, N, seed):
    g = gen(seed)
    C, F, L, R = 256, 512, 4, 16
    up, down = cci.pack(normal(g, 2 * F, C, std=0.1), 16, 4), cci.pack(normal(g, C, F, std=0.1), 16, 4)
    return dict(x=normal(g, N, C, dt=BF16), gamma=normal(g, C) * 0.1 + 1, beta=normal(g, C), up=up, down=down,
                A=normal(g, L, R, F, dt=BF16, std=0.05), B=normal(g, L, C, R, dt=BF16, std=0.2),
                rows=torch.randint(-1, L, (N,), generator=g, device=DEV, dtype=torch.int32),
                dout=normal(g, N, C, dt=BF16))


@pytest.mark.parametrize("N", [1, 77, 300])
def test_block_forward_and_backward(cci, N):
    s = block_state(cci, N, N)
    out, dx, dg, db, dv_up, dv_down = block(cci, s, True)
    served, = block(cci, s, False)
    # the same in 64 bits, with autograd
    dense = lambda vi: torch.zeros((vi[0].shape[0], 16, vi[0].shape[2]), dtype=F64, device=DEV).scatter_(  # noqa: E731
        1, vi[1].long(), vi[0].double()).view(-1, vi[0].shape[2])
    Wu, Wd = dense(s["up"]).requires_grad_(True), dense(s["down"]).requires_grad_(True)
    x, ga, be = s["x"].double().requires_grad_(True), s["gamma"].double().requires_grad_(True), s["beta"].double().requires_grad_(True)
    y = torch.nn.functional.layer_norm(x, (256,), ga, be)
    P = y @ Wu.t()
    h = torch.nn.functional.silu(P[:, :512]) * P[:, 512:]
    ref = h @ Wd.t()
    grads = torch.autograd.grad(ref, (x, ga, be, Wu, Wd), s["dout"].double())
    # bf16 between the operators: each of up to six roundings moves a value by 2^-8 of it at most; over a sum of random
    # signs the norm of the errors stays below six such steps of the result's norm
    far = lambda a, b: ((a.double() - b).norm() / b.norm()).item()  # noqa: E731
    lim = 6 * 2.0 ** -8
    assert far(out, ref + x) < lim
    for got, want in zip((dx, dg, db), grads[:3]):
        assert far(got, want) < lim
    for got, want, (_, idx) in ((dv_up, grads[3], s["up"]), (dv_down, grads[4], s["down"])):
        assert far(got, want.view(idx.shape[0], 16, -1).gather(1, idx.long())) < lim
    delta = torch.zeros_like(ref)
    for a in range(4):
        n = (s["rows"] == a).nonzero()[:, 0]
        delta[n] = (h[n] @ s["A"][a].double().t()) @ s["B"][a].double().t()
    assert far(served, ref + x + delta) < lim


@pytest.mark.parametrize("N", [3, 300])
def test_block_in_a_graph(cci, N):
    """Captured forward and backward, replayed on new inputs with eager work in between: equal bits; two graphs on
    streams of their own do not share workspaces."""
    s, t = block_state(cci, N, 1), block_state(cci, N, 2)
    want = {(k, train): [o.clone() for o in block(cci, v, train)] for k, v in (("s", s), ("t", t)) for train in (True, False)}
    side = torch.cuda.Stream()
    graphs = {}
    with torch.cuda.stream(side):
        for k, v in (("s", s), ("t", t)):
            block(cci, v, True), block(cci, v, False)
            side.synchronize()
            graphs[k] = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graphs[k], stream=side):
                graphs[k, "out"] = [block(cci, v, True), block(cci, v, False)]
    torch.cuda.synchronize()
    other = torch.cuda.Stream()
    for rep in range(4):
        with torch.cuda.stream(side):
            graphs["s"].replay()
        with torch.cuda.stream(other):
            graphs["t"].replay()
        torch.cuda.synchronize()
        eager = block(cci, s, True)
        for k in ("s", "t"):
            for train, outs in zip((True, False), graphs[k, "out"]):
                for a, b in zip(outs, want[k, train]):
                    assert torch.equal(a, b), (k, train, rep)
        for a, b in zip(eager, want["s", True]):
            assert torch.equal(a, b)
        for o in graphs["s", "out"][0]:
            o.zero_()
        torch.cuda.synchronize()


def test_equal_calls_give_equal_bits(cci):
    s = block_state(cci, 515, 3)
    first = [o.clone() for o in block(cci, s, True) + block(cci, s, False)]
    for _ in range(3):
        for a, b in zip(block(cci, s, True) + block(cci, s, False), first):
            assert torch.equal(a, b)


def test_other_stream(cci):
    s = block_state(cci, 130, 4)
    want = [o.clone() for o in block(cci, s, True) + block(cci, s, False)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = block(cci, s, True) + block(cci, s, False)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_two_streams_at_once(cci):
    """Calls in flight together have workspaces of their own."""
    states = [block_state(cci, n, 6 + n) for n in (515, 700)]
    want = [[o.clone() for o in block(cci, s, True) + block(cci, s, False)] for s in states]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in states]
    for _ in range(3):
        got = []
        for s, q in zip(states, streams):
            with torch.cuda.stream(q):
                got.append(block(cci, s, True) + block(cci, s, False))
        torch.cuda.synchronize()
        for g, w in zip(got, want):
            for a, b in zip(g, w):
                assert torch.equal(a, b)


# ------------------------------------------------- offsets past 32 bits --

def test_long_layernorm(cci):
    """4.3e9 elements: 1000 rows again and again, whose results are equal in every place."""
    g, C, reps = gen(70), 8192, 530
    X, dY, gamma = normal(g, 1000, C, dt=BF16), normal(g, 1000, C, dt=BF16), normal(g, C)
    y0, m0, r0 = cci.layernorm(X, gamma)
    d0, dg0, db0 = cci.layernorm_bwd(dY, X, m0, r0, gamma)
    Xs, dYs = X.repeat(reps, 1), dY.repeat(reps, 1)
    assert Xs.numel() > 2 ** 32
    y, m, r = cci.layernorm(Xs, gamma)
    d, dg, db = cci.layernorm_bwd(dYs, Xs, m, r, gamma)
    for long, short in ((y, y0), (m, m0), (r, r0), (d, d0)):
        assert (long.view(reps, *short.shape) == short).all()
    # the sums: 1000 terms of reps equal ones, N u S with S the terms' magnitudes (and those of the short sums)
    xh = ((X.double() - m0.double()[:, None]) * r0.double()[:, None])
    for got, terms in ((dg, dY.double() * xh), (db, dY.double())):
        within(got, reps * terms.sum(0), reps * terms.abs().sum(0) * (1000 * reps + 8) * U, "sums")


@pytest.mark.parametrize("G,K,C", [(8, 1, 64), (4, 1, 61)])
def test_long_products(cci, G, K, C):
    """Rows of 8192 past element 2^32: the last thousand rows give what a thousand alone do."""
    g, O, reps, B = gen(71), 8192, 530, 1000
    F = O // 2
    vals, idx, W = packed(cci, g, O, C, G, K, BF16)
    X, dH = normal(g, B, C, dt=BF16), normal(g, B, F, dt=BF16)
    Xs = X.repeat(reps, 1)
    H, pre = cci.gated_spmm(Xs, vals, idx, G, act="silu", save_pre=True)
    assert pre.numel() > 2 ** 32
    P, S, ref, a = gated_ref(X, W, F, "silu")
    e = (C + 2) * U * S
    slack = 1.2 * e[:, :F] * (P[:, F:].abs() + e[:, F:]) + a.abs() * e[:, F:] + 16 * U * P[:, :F].abs() * P[:, F:].abs()
    for k in (0, reps // 2, reps - 1):
        rows = slice(B * k, B * (k + 1))
        within(pre[rows], P, HALF[BF16] * P.abs() + e * (1 + HALF[BF16]), "pre")
        within(H[rows], ref, HALF[BF16] * ref.abs() + slack * (1 + HALF[BF16]), "H")
    dHs = dH.repeat(reps, 1)
    dpre, dX, dv = cci.gated_spmm_bwd(dHs, pre, Xs, vals, idx, G, act="silu", dvals_dtype=F32)
    assert (dpre.view(reps, B, O) == dpre[:B]).all()
    d = dpre[:B].double()
    for k in (0, reps - 1):
        check_product(dX[B * k:B * (k + 1)], d, W, O, "dX")
    x = X.double()
    ref, mag = reps * (d.t() @ x), reps * (d.abs().t() @ x.abs())
    at = idx.long()
    take = lambda t: t.view(O // G, G, C).gather(1, at)
    within(dv, take(ref), take(mag) * (B * reps + 8) * U, "dvals")
    del dpre, dX, pre, H, dHs
    L, R = 3, 5
    A, Bw = normal(g, L, R, C, dt=BF16), normal(g, L, O, R, dt=BF16)
    rows = torch.randint(-1, L, (B,), generator=g, device=DEV, dtype=torch.int32)
    short = cci.spmm_adapters(X, vals, idx, G, A, Bw, rows)
    Y = cci.spmm_adapters(Xs, vals, idx, G, A, Bw, rows.repeat(reps))
    # (both within the bound of the short product; the kernels may differ with the number of rows)
    w = W
    T = torch.einsum("nrc,nc->nr", A.double()[rows.clamp_min(0).long()], x) * (rows >= 0).double()[:, None]
    low = torch.einsum("nor,nr->no", Bw.double()[rows.clamp_min(0).long()], T)
    Tm = torch.einsum("nrc,nc->nr", A.double()[rows.clamp_min(0).long()].abs(), x.abs())
    lowm = torch.einsum("nor,nr->no", Bw.double()[rows.clamp_min(0).long()].abs(), Tm)
    want, mags = x @ w.t() + low, x.abs() @ w.abs().t() + lowm
    # D rounded once (2^-8), Y once; T enters with 16 bits (2^-16 of it), sums C + R terms
    tol = HALF[BF16] * (want.abs() + 1.01 * low.abs()) * 1.01 + mags * ((C + R + 8) * U + 2.0 ** -16)
    for got in (short, Y[:B], Y[-B:]):
        within(got, want, tol, "adapters")
