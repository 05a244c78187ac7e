"""RMS norm of residual streams, its int8 output and its gradients, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as R
from operators_testlib import DEV, HALF, T, U, Guarded, normal, np32, np64, replayed

pytestmark = pytest.mark.gpu
EPS = 1e-5

# (L, B, d): one row; odd batches; widths around every way the kernels cut a row; several layers; very wide rows
SHAPES = [(1, 1, 8), (1, 1, 2048), (3, 5, 64), (2, 33, 264), (1, 67, 512), (2, 19, 520), (1, 130, 768), (2, 31, 1024), (1, 9, 2056), (1, 21, 4096),
          (1, 5, 8200), (1, 3, 16384), (1, 2, 40008), (5, 257, 72)]


def sums_bound(d):
    """Relative error of a sum of d non-negative fp32 products added in any of the kernels' orders (a lane adds at most d / 64 of
    them, then a tree) and of the few operations after it."""
    return (d / 64 + 24) * U


def inputs(L, B, d, dtype, residual, seed=0):
    x = (normal(seed + 1, L, B, d) * torch.exp(0.5 * normal(seed + 2, L, B, 1))).to(T[dtype])
    r = (0.5 * normal(seed + 3, L, B, d)).to(T[dtype]) if residual else None
    w = 1.0 + 0.3 * normal(seed + 4, L, d)
    return x, r, w


def check_forward(x, r, w, dtype, h, y, q, scale, rstd):
    d = x.shape[-1]
    want_h, want_r, want_y = R.rms_norm(np32(x), np64(w), EPS, None if r is None else np32(r), dtype == "bf16")
    if h is not None:
        assert np.array_equal(np32(h), want_h)
    b = sums_bound(d)
    if rstd is not None:
        assert np.all(np.abs(np64(rstd) / want_r - 1) <= b)
    if y is not None:
        assert np.all(np.abs(np64(y) - want_y) <= np.abs(want_y) * (HALF[dtype] + b) * (1 + 2.0 ** -7) + 1e-38)
    if q is not None:
        top = np.abs(want_y).max(-1)
        t = want_h.astype(np.float64) * np64(w)[:, None, :]
        at = 127.0 * t / np.abs(t).max(-1, keepdims=True)
        # codes: rounded to nearest but for five fp32 roundings: of h w, the largest |h w|, its reciprocal, that times 127, the product
        assert np.all(np.abs(np64(q) - at) <= 0.5 + 127 * 5 * U)
        assert np.all(np.abs(np64(scale) / (top / 127.0) - 1) <= b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,B,d", SHAPES)
def test_forward(dtype, L, B, d):
    from paper_2603_21014_amd import binding as K
    for residual, native, int8 in ((True, True, True), (False, True, False), (True, False, True), (False, False, True)):
        x, r, w = inputs(L, B, d, dtype, residual)
        h = Guarded((L, B, d), T[dtype]) if residual else None
        y = Guarded((L, B, d), T[dtype]) if native else None
        q, scale = (Guarded((L, B, d), torch.int8), Guarded((L, B), torch.float32)) if int8 else (None, None)
        rstd = Guarded((L, B), torch.float32)
        t = lambda g: g.t if g else None
        K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=t(y), q=t(q), q_scale=t(scale), residual=r.to(DEV) if residual else None, h=t(h),
                       rstd=rstd.t if native else None)
        torch.cuda.synchronize()
        check_forward(x, r, w, dtype, t(h), t(y), t(q), t(scale), rstd.t if native else None)
        for g in (h, y, q, scale, rstd):
            if g:
                g.check()


def test_sum_in_place_of_either_operand():
    from paper_2603_21014_amd import binding as K
    x, r, w = inputs(2, 37, 520, "bf16", True)
    for into in (0, 1):
        xd, rd = x.to(DEV), r.to(DEV)
        y = torch.empty_like(xd)
        K.clt_rms_norm(xd, w.to(DEV), EPS, y=y, residual=rd, h=(xd, rd)[into])
        check_forward(x, r, w, "bf16", (xd, rd)[into], y, None, None, None)
        assert torch.equal((rd, xd)[into].cpu(), (r, x)[into])


def test_special_rows():
    """Rows of zeros, of denormals, with an infinity, with a NaN, with the type's largest values, of one non-zero element."""
    from paper_2603_21014_amd import binding as K
    for dtype in ("bf16", "f32"):
        x = normal(5, 1, 7, 264).to(T[dtype])
        x[0, 0] = 0.0
        x[0, 1] = 1e-40
        x[0, 2, 100] = float("inf")
        x[0, 3, 263] = float("nan")
        x[0, 4] = 0.0
        x[0, 4, 200] = -3.0
        x[0, 5] = 1e18
        w = torch.ones(1, 264)
        y, q = torch.empty_like(x, device=DEV), torch.full((1, 7, 264), 77, dtype=torch.int8, device=DEV)
        s, rstd = torch.empty(1, 7, device=DEV), torch.empty(1, 7, device=DEV)
        K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=y, q=q, q_scale=s, rstd=rstd)
        q, s, y = q.cpu()[0], s.cpu()[0], y.float().cpu()[0]
        for row in (0, 1):
            assert not q[row].any() and s[row] == 1.0 and torch.all(y[row].abs() < 1e-30)
        for row in (2, 3):
            assert not q[row].any() and torch.isnan(s[row])
        assert torch.isnan(y[3]).all() and torch.isnan(y[2, 100]) and not y[2, :100].any()
        assert q[4, 200] == -127 and not q[4, :200].any() and s[4] > 0
        assert torch.all(q[5] == 127) and abs(float(s[5]) * 127 - 1) < 1e-5
        check_forward(x[:, 6:], None, w, dtype, None, None, q[None, 6:], s[None, 6:], None)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,B,d", SHAPES)
def test_backward(dtype, L, B, d):
    from paper_2603_21014_amd import binding as K
    for residual in (False, True):
        x, e, w = inputs(L, B, d, dtype, residual, seed=10)
        dy = normal(20, L, B, d).to(T[dtype])
        rstd = torch.from_numpy(R.rms_norm(np32(x), np64(w), EPS)[1]).float()
        dx, dw = Guarded((L, B, d), T[dtype]), Guarded((L, d), torch.float32)
        n = K.clt_rms_norm_backward_workspace_bytes(L, B, d)
        ws = Guarded((n,), torch.uint8)
        K.clt_rms_norm_backward(x.to(DEV), w.to(DEV), rstd.to(DEV), dy.to(DEV), dx.t, dw.t, ws.t, dh=e.to(DEV) if residual else None)
        torch.cuda.synchronize()
        want_dx, want_dw = R.rms_norm_backward(np32(x), np64(w), np64(rstd), np32(dy), None if e is None else np32(e))
        h, g, r = np64(x), np64(dy), np64(rstd)[..., None]
        wg = np.abs(np64(w)[:, None, :] * g)
        size = r * wg + np.abs(h) * r ** 3 * (wg * np.abs(h)).mean(-1, keepdims=True) + (0 if e is None else np.abs(np64(e)))
        assert np.all(np.abs(np64(dx.t) - want_dx) <= HALF[dtype] * np.abs(want_dx) + size * sums_bound(d) * 1.01 + 1e-38)
        assert np.all(np.abs(np64(dw.t) - want_dw) <= (np.abs(g * h * r)).sum(1) * (B + 8) * U)
        for guard in (dx, dw, ws):
            guard.check()
        # without the weights' gradient, in place of dy and of dh, and again: the same bits
        again = dy.to(DEV)
        K.clt_rms_norm_backward(x.to(DEV), w.to(DEV), rstd.to(DEV), again, again, dh=e.to(DEV) if residual else None)
        assert torch.equal(again, dx.t)
        if residual:
            over, dw2 = e.to(DEV), torch.empty_like(dw.t)
            K.clt_rms_norm_backward(x.to(DEV), w.to(DEV), rstd.to(DEV), dy.to(DEV), over, dw2, ws.t, dh=over)
            assert torch.equal(over, dx.t) and torch.equal(dw2, dw.t)


def test_gradients_against_differences():
    """Forward and backward pass together, in fp32: a change of the inputs along a direction changes sum(y g) by the gradient's
    product with it.  Step 2^-6 in a function whose third derivative is of order one: 2^-12 / 6 of the largest terms, plus
    rounding 2^-24 * sqrt(n) / 2^-6."""
    from paper_2603_21014_amd import binding as K
    L, B, d = 2, 9, 264
    x, _, w = inputs(L, B, d, "f32", False, seed=30)
    g, ux, uw = normal(41, L, B, d), normal(42, L, B, d), normal(43, L, d)

    def value(x, w):
        y = torch.empty_like(x, device=DEV)
        K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=y)
        return float((y.double().cpu() * g.double()).sum())
    rstd, y, dx = torch.empty(L, B, device=DEV), torch.empty(L, B, d, device=DEV), torch.empty(L, B, d, device=DEV)
    dw = torch.empty(L, d, device=DEV)
    K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=y, rstd=rstd)
    ws = torch.empty(K.clt_rms_norm_backward_workspace_bytes(L, B, d), dtype=torch.uint8, device=DEV)
    K.clt_rms_norm_backward(x.to(DEV), w.to(DEV), rstd, g.to(DEV), dx, dw, ws)
    s = 2.0 ** -6
    for along, got in (((value(x + s * ux, w) - value(x - s * ux, w)) / (2 * s), (dx.double().cpu() * ux.double()).sum()),
                       ((value(x, w + s * uw) - value(x, w - s * uw)) / (2 * s), (dw.double().cpu() * uw.double()).sum())):
        assert abs(along - float(got)) <= 3e-3 * np.sqrt(L * B * d), (along, float(got))


def test_streams_and_graphs():
    from paper_2603_21014_amd import binding as K
    L, B, d = 2, 300, 520
    x, r, w = (t.to(DEV) for t in inputs(L, B, d, "bf16", True, seed=50))
    h, q = torch.empty_like(x), torch.empty(L, B, d, dtype=torch.int8, device=DEV)
    s, rstd, dx, dw = torch.empty(L, B, device=DEV), torch.empty(L, B, device=DEV), torch.empty_like(x), torch.empty(L, d, device=DEV)
    ws = torch.empty(K.clt_rms_norm_backward_workspace_bytes(L, B, d), dtype=torch.uint8, device=DEV)

    def call():
        K.clt_rms_norm(x, w, EPS, q=q, q_scale=s, residual=r, h=h, rstd=rstd)
        K.clt_rms_norm_backward(h, w, rstd, r, dx, dw, ws, dh=x)
    call()
    want = [t.clone() for t in (h, q, s, rstd, dx, dw)]
    for got in replayed(call, (h, q, s, rstd, dx, dw)):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((h, q, s, rstd, dx, dw), want))


def test_codes_are_what_the_step_reads():
    """The encoder on the int8 codes and scales of the norm against the one on the native norm: the same pre-activations up to
    the codes' rounding."""
    from paper_2603_21014_amd import binding as K
    L, B, d, F = 2, 65, 264, 136
    x, r, w = (t.to(DEV) for t in inputs(L, B, d, "bf16", True, seed=60))
    h, y, q, s = torch.empty_like(x), torch.empty_like(x), torch.empty(L, B, d, dtype=torch.int8, device=DEV), torch.empty(L, B, device=DEV)
    K.clt_rms_norm(x, w, EPS, y=y, q=q, q_scale=s, residual=r, h=h)
    g = torch.Generator(device=DEV).manual_seed(1)
    params = {"W_enc": (torch.randn((L, d, F), generator=g, device=DEV) / d ** 0.5).bfloat16(), "b_enc": torch.zeros(L, F, device=DEV),
              "theta": torch.full((L, F), 0.03, device=DEV), "W_dec": torch.zeros(3, F, d, dtype=torch.bfloat16, device=DEV),
              "b_dec": torch.zeros(L, d, device=DEV)}
    step = K.CLTStep(L, d, F, B, int8_inputs=True, device=DEV)
    step.forward(q, params, s)
    exact = torch.matmul((q.double() * s.double()[..., None]), params["W_enc"].double())
    assert torch.all((step.pre.double() - exact).abs() <= 2.0 ** -8 * exact.abs() + 1e-5)
    native = torch.matmul(y.double(), params["W_enc"].double())
    # codes off by half a step of s, y by half a step of bf16, d terms of random signs: five deviations
    sigma = ((s.double() ** 2 / 12)[..., None] * d + (y.double() ** 2).sum(-1, keepdim=True) * 2.0 ** -16 / 3).sqrt() / d ** 0.5
    assert torch.all((exact - native).abs() <= 6 * sigma)


def test_binding_refusals_on_the_device():
    from paper_2603_21014_amd import binding as K
    x, w = torch.zeros(2, 4, 64, device=DEV), torch.ones(2, 64, device=DEV)
    y = torch.full_like(x, 5.0)
    for bad in (lambda: K.clt_rms_norm(x, w[:1], EPS, y=y), lambda: K.clt_rms_norm(x, w, EPS, y=y[:, :3]),
                lambda: K.clt_rms_norm(x.transpose(1, 2), w, EPS, y=y), lambda: K.clt_rms_norm(x, w, EPS, y=y.bfloat16()),
                lambda: K.clt_rms_norm(x, w.cpu(), EPS, y=y), lambda: K.clt_rms_norm_backward(x, w, x[..., 0].contiguous(), x, y, workspace=w)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: K.clt_rms_norm(x, w, EPS), lambda: K.clt_rms_norm(x, w, 0.0, y=y), lambda: K.clt_rms_norm(x, w, EPS, y=y, residual=x),
                lambda: K.clt_rms_norm_backward(x, w, x[..., 0].contiguous(), x, y, torch.empty_like(w)),
                lambda: K.clt_rms_norm(x[:, :, :60].contiguous(), w[:, :60].contiguous(), EPS, y=y[:, :, :60].contiguous())):
        with pytest.raises(K.CLTError):
            bad()
    torch.cuda.synchronize()
    assert torch.all(y == 5.0)


# Rows whose squares, or whose products with the weights, are beyond fp32: every width that the kernels cut differently
LARGE = [("bf16", 264), ("bf16", 776), ("bf16", 2048), ("bf16", 2056), ("bf16", 8192), ("bf16", 8200), ("f32", 136), ("f32", 1024), ("f32", 1032), ("f32", 4096), ("f32", 4104)]
POWERS = (0, 30, 45, 58, 61, 63, 64, 65, 80, 100, 120, 124)


def large_rows(dtype, d, seed):
    """[2, 15, d]: normal numbers times powers of two; the type's largest number throughout, and once among ordinary ones; ordinary again."""
    x = normal(seed, 2, len(POWERS) + 3, d)
    x[:, :len(POWERS)] *= torch.tensor([2.0 ** k for k in POWERS])[:, None]
    x = x.to(T[dtype])
    top = torch.finfo(T[dtype]).max
    x[:, len(POWERS)] = torch.where(normal(seed + 1, 2, d) > 0, top, -top).to(T[dtype])
    x[:, len(POWERS) + 1, d // 3] = -top
    return x, 1.0 + 0.3 * normal(seed + 2, 2, d)


@pytest.mark.parametrize("dtype,d", LARGE)
def test_rows_of_very_large_numbers(dtype, d):
    from paper_2603_21014_amd import binding as K
    x, w = large_rows(dtype, d, 70)
    L, B, _ = x.shape
    r = (x.float() * 0.25).to(T[dtype])
    r[:, len(POWERS):len(POWERS) + 2] = 0.0      # (the sum of these stays finite)
    for residual in (None, r):
        h = torch.empty_like(x, device=DEV) if residual is not None else None
        y, q = torch.empty_like(x, device=DEV), torch.empty(L, B, d, dtype=torch.int8, device=DEV)
        s, rstd = torch.empty(L, B, device=DEV), torch.empty(L, B, device=DEV)
        K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=y, q=q, q_scale=s, residual=None if residual is None else residual.to(DEV), h=h, rstd=rstd)
        assert torch.isfinite(y).all() and torch.isfinite(s).all() and q.any(-1).all()
        check_forward(x, residual, w, dtype, h, y, q, s, None)
        want = R.rms_norm(np32(x), np64(w), EPS, None if residual is None else np32(residual), dtype == "bf16")[1]
        assert np.all(np.abs(np64(rstd) - want) <= sums_bound(d) * want + 2.0 ** -149)      # (half a step of the smallest numbers, twice)
    # a row with an infinity beside large numbers is still a broken one, and no row depends on another
    again = x.clone()
    again[:, 3, d - 1], again[:, 9, 0] = float("inf"), float("nan")
    y2, q2, s2 = torch.empty_like(y), torch.empty_like(q), torch.empty_like(s)
    K.clt_rms_norm(again.to(DEV), w.to(DEV), EPS, y=y2, q=q2, q_scale=s2)
    K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=y, q=q, q_scale=s)
    for b in range(B):
        if b in (3, 9):
            assert torch.isnan(s2[:, b]).all() and not q2[:, b].any()
        else:
            assert torch.equal(y[:, b], y2[:, b]) and torch.equal(q[:, b], q2[:, b]) and torch.equal(s[:, b], s2[:, b])


@pytest.mark.parametrize("dtype,d", LARGE)
def test_gradients_of_rows_of_very_large_numbers(dtype, d):
    from paper_2603_21014_amd import binding as K
    x, w = large_rows(dtype, d, 80)
    L, B, _ = x.shape
    rstd = torch.from_numpy(R.rms_norm(np32(x), np64(w), EPS)[1]).float()
    dy, e = (4.0 * normal(83, L, B, d)).to(T[dtype]), (2.0 ** -90 * normal(84, L, B, d)).to(T[dtype])
    ws = torch.empty(K.clt_rms_norm_backward_workspace_bytes(L, B, d), dtype=torch.uint8, device=DEV)
    for dh in (None, e):
        dx, dw = torch.empty_like(x, device=DEV), torch.empty(L, d, device=DEV)
        K.clt_rms_norm_backward(x.to(DEV), w.to(DEV), rstd.to(DEV), dy.to(DEV), dx, dw, ws, dh=None if dh is None else dh.to(DEV))
        want_dx, want_dw = R.rms_norm_backward(np32(x), np64(w), np64(rstd), np32(dy), None if dh is None else np32(dh))
        h, g, r = np64(x), np64(dy), np64(rstd)[..., None]
        wg = np.abs(np64(w)[:, None, :] * g)
        size = r * wg + np.abs(h) * r ** 3 * (wg * np.abs(h)).mean(-1, keepdims=True) + (0 if dh is None else np.abs(np64(dh)))
        # (1e-38: results among the smallest numbers, where a step is not relative to the value)
        assert np.all(np.abs(np64(dx) - want_dx) <= HALF[dtype] * np.abs(want_dx) + size * sums_bound(d) * 1.01 + 1e-38)
        assert np.all(np.abs(np64(dw) - want_dw) <= (np.abs(g * h * r)).sum(1) * (B + 8) * U)


@pytest.mark.parametrize("dtype,d", LARGE)
def test_rows_under_very_large_weights(dtype, d):
    """Rows of one size throughout, whose norm is 1, so that y is the weight: finite, while h weight is not."""
    from paper_2603_21014_amd import binding as K
    powers = (0, 1, 10, 53, 70, 126, 127)
    sign = torch.where(normal(90, 1, len(powers), d) > 0, 1.0, -1.0)
    x = (sign * torch.tensor([1.9375 * 2.0 ** k for k in powers])[:, None]).to(T[dtype])      # (5 bits: exact in bf16)
    w = torch.full((1, d), 3e38) * (1 - 0.25 * torch.rand((1, d), generator=torch.Generator().manual_seed(91)))
    y, q = torch.empty_like(x, device=DEV), torch.empty(1, len(powers), d, dtype=torch.int8, device=DEV)
    s = torch.empty(1, len(powers), device=DEV)
    K.clt_rms_norm(x.to(DEV), w.to(DEV), EPS, y=y, q=q, q_scale=s)
    assert torch.isfinite(y).all() and torch.isfinite(s).all() and (q != 0).all()
    check_forward(x, None, w, dtype, None, y, q, s, None)
