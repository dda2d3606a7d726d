"""Outputs of the feed-forward block's operators held to the rounding that
their definitions leave, where a looser bound would pass a wrong step.

Tolerances are those of test_gpu_block.py: u = 2^-24 per term of an fp32 sum,
half a step of the output's type for its one rounding.
"""
import ctypes
import math

import pytest
import torch

from gpu_common import DEV, Guarded
from test_gpu_block import ACTS, BF16, F32, F64, HALF, U, cci, gen, normal, packed, within  # noqa: F401

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- adapters --

def adapter_terms(X, W, A, B, rows, alpha):
    """Product, adapters' term, and the magnitudes of the terms of either, in 64 bits."""
    x = X.double()
    acc, S = x @ W.t(), x.abs() @ W.abs().t()
    D, SD = torch.zeros_like(acc), torch.zeros_like(acc)
    for a in range(A.shape[0]):
        n = (rows == a).nonzero()[:, 0]
        f = alpha[a].double()
        D[n] = f * (x[n] @ A[a].double().t()) @ B[a].double().t()
        SD[n] = f.abs() * (x[n].abs() @ A[a].double().abs().t()) @ B[a].double().abs().t()
    return acc, S, D, SD


def check_adapters(got, X, W, A, B, rows, alpha, res, relu, what):
    """One rounding to the output's type: T enters a bf16 product in two parts (2^-16 of each term), the three terms
    are added in fp32 (u of each partial sum)."""
    C, R = X.shape[1], A.shape[1]
    acc, S, D, SD = adapter_terms(X, W, A, B, rows, alpha)
    r = res.double()
    ref = acc + r + D
    e = ((C + 8) * U * S + ((C + R + 24) * U + (2.0 ** -16 if X.dtype == BF16 else 0.0)) * SD
         + 4 * U * (S + SD + r.abs()))
    if relu:
        ref = ref.clamp_min(0)
    within(got, ref, HALF[got.dtype] * ref.abs() + e * (1 + HALF[got.dtype]), what)


@pytest.mark.parametrize("dt,y_t", [(BF16, BF16), (BF16, F32), (F32, F32)], ids=["bf16", "bf16-f32", "f32"])
@pytest.mark.parametrize("size", [(1, 256, 256, 16, 4, 3, 16), (40, 512, 256, 16, 4, 5, 16), (200, 256, 264, 8, 2, 4, 32),
                                  (333, 129, 48, 4, 1, 7, 33), (70, 320, 66, 3, 2, 3, 8)])
def test_adapters_round_once(cci, size, dt, y_t):  # noqa: F811
    N, C, O, G, K, L, R = size
    g = gen(N)
    X, A, B = normal(g, N, C, dt=dt), normal(g, L, R, C, dt=dt, std=C ** -0.5), normal(g, L, O, R, dt=dt, std=R ** -0.5)
    vals, idx, W = packed(cci, g, O, C, G, K, dt)
    rows = torch.randint(-1, L, (N,), generator=g, device=DEV, dtype=torch.int32)
    alpha = 1 + normal(g, L, std=0.1)
    # a residual that all but cancels the other terms: what was rounded before the sum would stand out
    acc, _, D, _ = adapter_terms(X, W, A, B, rows, alpha)
    for res, relu in ((normal(g, N, O, dt=y_t, std=4.0), False), ((-(acc + D)).to(y_t), False), (normal(g, N, O, dt=y_t), True)):
        out = Guarded((N, O), y_t)
        got = cci.spmm_adapters(X, vals, idx, G, A, B, rows, alpha=alpha, residual=res, relu=relu, out_dtype=y_t, out=out.t)
        torch.cuda.synchronize()
        check_adapters(got, X, W, A, B, rows, alpha, res, relu, f"relu {relu}")
        out.check("adapters")
        # the residual may be the output
        same = res.clone()
        cci.spmm_adapters(X, vals, idx, G, A, B, rows, alpha=alpha, residual=same, relu=relu, out_dtype=y_t, out=same)
        assert torch.equal(same, got)


def test_adapters_in_slices_of_rows(cci):  # noqa: F811
    """Outputs so wide that a call's rows go through the workspace in two slices."""
    N, C, O, G, K, L, R = 300, 8, 1 << 20, 8, 2, 3, 4
    g = gen(1)
    X, A, B = normal(g, N, C, dt=BF16), normal(g, L, R, C, dt=BF16), normal(g, L, O, R, dt=BF16, std=0.5)
    vals, idx, W = packed(cci, g, O, C, G, K, BF16)
    rows = torch.randint(-1, L, (N,), generator=g, device=DEV, dtype=torch.int32)
    alpha, res = 1 + normal(g, L, std=0.1), normal(g, N, O, dt=BF16)
    out = Guarded((N, O), BF16)
    cci.spmm_adapters(X, vals, idx, G, A, B, rows, alpha=alpha, residual=res, out=out.t)
    torch.cuda.synchronize()
    for n in range(0, N, 50):
        s = slice(n, n + 50)
        check_adapters(out.t[s], X[s], W, A, B, rows[s], alpha, res[s], False, f"rows {n}")
    out.check("adapters")


# -------------------------------------------------------------- layer norm --

@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("C", [1, 40, 1500, 16392])
@pytest.mark.parametrize("eps", [1e-5, 0.0])
def test_layernorm_statistics_of_non_finite_rows(cci, C, dt, eps):  # noqa: F811
    """mean and rstd are the formulas' for rows that hold infinities or NaN, and the other rows' stay."""
    inf, nan = float("inf"), float("nan")
    X = (normal(gen(C), 6, C) + 1).to(dt)
    clean = X.clone()
    for n, v in ((1, inf), (2, -inf), (4, nan)):
        X[n, C // 2] = v
    if C > 1:
        X[5, 0], X[5, C - 1] = inf, -inf
    Y, mean, rstd = cci.layernorm(X, eps=eps)
    want = X.double().mean(1)
    assert mean[1] == inf and mean[2] == -inf and mean[4].isnan()
    for n in (1, 2, 4) + ((5,) if C > 1 else ()):
        assert torch.equal(mean[n].isnan(), want[n].isnan()) and rstd[n].isnan() and Y[n].isnan().all(), n
    for got, alone in zip((Y, mean, rstd), cci.layernorm(clean, eps=eps)):
        for n in (0, 3):
            assert torch.equal(got[n].isnan(), alone[n].isnan()) and torch.equal(got[n].nan_to_num(7), alone[n].nan_to_num(7))


@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("C", [776, 4096, 16392])
def test_layernorm_mean_is_as_good_as_a_sum(cci, C, dt):  # noqa: F811
    """Means of rows of deviation 1, on average over 2000 rows.  A sum in fp32 whose partial sums grow as sqrt(k) (k up
    to 64 in a thread, then 10 levels that each hold C terms in all) is off by u / sqrt(3) of every partial sum, at
    random: by less than u sqrt((32 + 10) C / 3) in all, 3.8 u / sqrt(C) of the mean.  The mean's own rounding adds half
    a step of it, u |m| at most; deviations that lose the same part for every x would add up to u."""
    X = (normal(gen(C), 2000, C) + normal(gen(C + 1), 2000, 1, std=0.1)).to(dt)
    mean = cci.layernorm(X)[1].double()
    want = X.double().mean(1)
    off = (mean - want).abs().mean().item()
    assert off <= U * (3.8 / C ** 0.5 + want.abs().mean().item()), off / U


@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("N,C", [(5, 40), (70, 1001), (9, 4096), (3, 16384), (3, 16392), (700, 16393)])
def test_layernorm_bwd_in_parts(cci, N, C, dt):  # noqa: F811
    """The gradients that are wanted are those of the whole call; without the weights' nothing is written to the
    workspace, which need not be there for rows of up to 16384."""
    g = gen(N + C)
    X, dY, gamma = normal(g, N, C, dt=dt), normal(g, N, C, dt=dt), normal(g, C) + 1
    _, mean, rstd = cci.layernorm(X, gamma)
    whole = cci.layernorm_bwd(dY, X, mean, rstd, gamma)
    dX, dg, db = cci.layernorm_bwd(dY, X, mean, rstd, gamma, need_dw=False)
    assert dg is None and db is None and torch.equal(dX, whole[0])
    dX, dg, db = cci.layernorm_bwd(dY, X, mean, rstd, gamma, need_dx=False)
    assert dX is None and torch.equal(dg, whole[1]) and torch.equal(db, whole[2])
    assert cci.layernorm_bwd(dY, X, mean, rstd, gamma, need_dx=False, need_dw=False) == (None, None, None)
    nb = ctypes.c_size_t()
    assert cci.raw().cci_layernorm_bwd_workspace(N, C, ctypes.byref(nb)) == cci.OK
    out, ws = Guarded((N, C), dt), torch.full((nb.value,), 0x7f, dtype=torch.uint8, device=DEV)

    def call(dx, dgamma, dbeta, w):
        return cci.raw().cci_layernorm_bwd(dY.data_ptr(), X.data_ptr(), cci._code(dt), N, C, gamma.data_ptr(), mean.data_ptr(),
                                           rstd.data_ptr(), cci._ptr(dx), cci._ptr(dgamma), cci._ptr(dbeta), cci._ptr(w),
                                           0 if w is None else nb.value, None)

    assert call(out.t, None, None, ws) == cci.OK
    torch.cuda.synchronize()
    assert torch.equal(out.t, whole[0])
    sums = nb.value - (8 * N if C > 16384 else 0)  # (long rows keep two values each behind the sums)
    assert (ws[:sums] == 0x7f).all()
    if C <= 16384:
        assert call(out.t, None, None, None) == cci.OK
    else:
        assert call(out.t, None, None, None) == cci.EINVAL
    only = torch.empty(C, device=DEV)
    assert call(None, None, only, ws) == cci.OK
    assert torch.equal(only, whole[2])
    out.check("dX")


def test_layernorm_bwd_of_very_long_rows(cci):  # noqa: F811
    """Weight gradients of more columns than a launch has threads for, 16 to a column and kind."""
    C = (1 << 27) + 5
    g = gen(3)
    X, dY = normal(g, 1, C, dt=BF16), normal(g, 1, C, dt=BF16)
    mean, rstd = torch.tensor([0.25], device=DEV), torch.tensor([1.5], device=DEV)
    dX, dg, db = cci.layernorm_bwd(dY, X, mean, rstd)
    assert torch.equal(db, dY[0].float())
    want = dY[0].float() * ((X[0].float() - 0.25) * 1.5)
    assert torch.allclose(dg, want, rtol=8 * U, atol=0)  # three roundings either way
    q, xh = dY[0].double(), (X[0].double() - 0.25) * 1.5
    ref = 1.5 * (q - q.mean() - xh * (q * xh).mean())
    # a thread adds 2^14 terms, then 10 levels
    slack = 1.5 * (2 ** 14 + 10) * U * (q.abs().mean() + xh.abs() * (q * xh).abs().mean()) + 16 * U * (q.abs() + xh.abs())
    within(dX[0], ref, HALF[BF16] * ref.abs() + slack * (1 + HALF[BF16]), "dX")


# -------------------------------------------------------------- activations --

def act_parts(x, name):
    """act(x) and act'(x) in 64 bits without cancellation in the tails, the magnitudes of the slope's terms, and the
    size of the argument of the exponential in them."""
    if name == "gelu":
        # (torch.special.ndtr is 0 from -8.3 on, where Phi is 5e-17)
        c, q = torch.special.erfc(x * -0.5 ** 0.5) / 2, torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)
        return x * c, c + x * q, c + (x * q).abs(), x * x
    if name in ("silu", "gelu_tanh"):
        k = math.sqrt(8 / math.pi)
        z, dz = (x, 1.0) if name == "silu" else (k * (x + 0.044715 * x ** 3), k * (1 + 0.134145 * x * x))
        s, e = torch.sigmoid(z), torch.sigmoid(z) * torch.sigmoid(-z)
        return x * s, s + x * e * dz, s + (x * e * dz).abs(), z.abs()
    return (x.clamp_min(0), (x > 0).double(), (x > 0).double(), 0 * x) if name == "relu" else (x, torch.ones_like(x), torch.ones_like(x), 0 * x)


@pytest.mark.parametrize("dt", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
def test_activation_tails(cci, act, dt):  # noqa: F811
    """Values and slopes from -12 to 12 beside a large up value, relative to themselves.  An exponential's argument z
    comes with up to 6 u of its size, 16 u are the library functions' and 8 the products'; below 1e-35 they underflow."""
    F, up = 2048, 1000.0
    x = torch.linspace(-12, 12, F, device=DEV).to(dt)
    W = torch.cat((x.float(), torch.full((F,), up, device=DEV))).view(-1, 1)
    vals, idx = cci.pack(W, 1, 1, dt)
    X = torch.tensor([[1.0], [-1.0], [0.5]], device=DEV, dtype=dt)
    H, pre = cci.gated_spmm(X, vals, idx, 1, act=act, save_pre=True)
    p = X.double() * W.double().t()
    assert torch.equal(pre.double(), p)  # powers of two times values of the type
    g, u = p[:, :F], p[:, F:]
    a, d, terms, z = act_parts(g, act)
    rel = (6 * z + 24) * U
    within(H, a * u, (a * u).abs() * (HALF[dt] + rel) * (1 + HALF[dt]) + 1e-35 * up, "H")
    dH = torch.full_like(H, 3.0)
    dpre, _, _ = cci.gated_spmm_bwd(dH, pre, X, vals, idx, 1, act=act)
    within(dpre[:, F:], 3 * a, (3 * a).abs() * (HALF[dt] + rel) * (1 + HALF[dt]) + 1e-35, "du")
    within(dpre[:, :F], 3 * u * d, (3 * u * d).abs() * HALF[dt] + 3 * u.abs() * terms * rel * (1 + HALF[dt]) + 1e-35 * up, "dg")


@pytest.mark.parametrize("act", ACTS)
def test_activations_far_out(cci, act):  # noqa: F811
    """Arguments whose square or cube overflows: the activations are 0 or the argument there, their slopes 0 or 1."""
    g = torch.tensor([3e4, 1e20, 3e38, -3e4, -1e20, -3e38, 0.0], device=DEV)
    F = g.numel()
    vals, idx = cci.pack(torch.cat((g, torch.full((F,), 0.5, device=DEV))).view(-1, 1), 1, 1, F32)
    X = torch.ones((1, 1), device=DEV)
    H, pre = cci.gated_spmm(X, vals, idx, 1, act=act, save_pre=True)
    dpre, _, _ = cci.gated_spmm_bwd(torch.ones_like(H), pre, X, vals, idx, 1, act=act)
    none = act == "none"
    a = g if none else g.clamp_min(0)
    at0 = {"none": 1.0, "relu": 0.0}.get(act, 0.5)
    d = torch.where(g == 0, at0, ((g > 0) | none).float())
    assert torch.equal(H[0], 0.5 * a) and torch.equal(dpre[0, F:], a) and torch.equal(dpre[0, :F], 0.5 * d)


# -------------------------------------------------- more tiles than a launch --

@pytest.mark.parametrize("N,C,G", [(3, 1 << 18, 256), (33, 1 << 19, 128)])
def test_packed_gradient_of_a_very_large_layer(cci, N, C, G):  # noqa: F811
    """2^20 weight rows: the packed gradient has more tiles than one launch has threads for.  Samples of small whole
    numbers: every sum is exact."""
    F, K = 1 << 19, 1
    g = gen(N)
    idx = torch.randint(0, G, (2 * F // G, K, C), generator=g, device=DEV, dtype=torch.uint8)
    X = torch.randint(-2, 3, (N, C), generator=g, device=DEV).to(BF16)
    dH = torch.randint(-2, 3, (N, F), generator=g, device=DEV).to(BF16)
    pre = torch.randint(-2, 3, (N, 2 * F), generator=g, device=DEV).to(BF16)
    vals = torch.empty((2 * F // G, K, C), dtype=BF16, device=DEV)  # (not read without dX)
    dpre, _, dv = cci.gated_spmm_bwd(dH, pre, X, vals, idx, G, act="none", need_dx=False)
    d, x = dpre.float(), X.float()
    assert torch.equal(d, torch.cat((dH.float() * pre[:, F:].float(), dH.float() * pre[:, :F].float()), 1))
    groups, step = 2 * F // G, 64
    for lo in [*range(0, groups, step * (1 if N < 8 else 8)), groups - step]:
        rows = (torch.arange(lo, lo + step, device=DEV)[:, None] * G + idx[lo:lo + step, 0].long())
        want = torch.zeros((step, C), device=DEV)
        for n in range(N):
            want += d[n][rows] * x[n]
        assert torch.equal(dv[lo:lo + step, 0].float(), want.to(BF16).float()), lo
