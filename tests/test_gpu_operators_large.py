"""Operators around the training step on tensors of more than 2^32 elements: what lies behind that border is what the oracle says
of those elements alone."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as R
from operators_testlib import DEV, HALF, U, normal, np32, np64

pytestmark = pytest.mark.gpu
FAR = 1 << 32


@pytest.fixture(autouse=True)
def _room():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


def test_adamw_behind_2_to_the_32():
    from paper_2603_21014_amd import binding as K
    tail, n = 5003, FAR + 5003
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device=DEV)
    p, g, m, v = z(torch.bfloat16), z(torch.bfloat16), z(torch.uint8), z(torch.uint8)
    ms, vs = z(torch.uint8, (n + 127) // 128), z(torch.uint8, (n + 127) // 128)
    hp, hg = normal(1, tail).bfloat16(), (1e-3 * normal(2, tail)).bfloat16()
    p[FAR:], g[FAR:] = hp.to(DEV), hg.to(DEV)
    opt = K.AdamW([K.AdamWTensor(p, g, m, v, ms, vs)], seed=99)
    hm, hv = np.zeros(tail, np.uint8), np.zeros(tail, np.uint8)
    hms, hvs = np.zeros(-(-tail // 128), np.uint8), np.zeros(-(-tail // 128), np.uint8)
    real = R.random_bits
    try:
        R.random_bits = lambda seed, t, index, k: real(seed, t, index, k, first=FAR)
        for t in (1, 2):
            opt.step(t, 1e-3)
            torch.cuda.synchronize()
            o = R.adamw(np.zeros(tail), np32(hg), hm, hv, t, 1e-3, 0.9, 0.999, 1e-8, 0.0, hms, hvs, 99, 0)
            hm, hv, hms, hvs = o["m"], o["v"], o["m_scale"], o["v_scale"]
            assert np.array_equal(m[FAR:].cpu().numpy(), hm) and np.array_equal(v[FAR:].cpu().numpy(), hv)
            assert np.array_equal(ms[FAR // 128:].cpu().numpy(), hms) and np.array_equal(vs[FAR // 128:].cpu().numpy(), hvs)
    finally:
        R.random_bits = real
    assert not m[:FAR].any() and not p[:FAR].any()      # no gradient: nothing moves


def test_rms_norm_and_gradients_behind_2_to_the_32():
    from paper_2603_21014_amd import binding as K
    d, B = 2048, (FAR // 2048) + 70
    x, dy = torch.zeros(1, B, d, dtype=torch.bfloat16, device=DEV), torch.zeros(1, B, d, dtype=torch.bfloat16, device=DEV)
    hx, hg, w = normal(3, 1, 70, d).bfloat16(), normal(4, 1, 70, d).bfloat16(), 1 + 0.1 * normal(5, 1, d)
    x[:, -70:], dy[:, -70:] = hx.to(DEV), hg.to(DEV)
    q, s, rstd = torch.empty(1, B, d, dtype=torch.int8, device=DEV), torch.empty(1, B, device=DEV), torch.empty(1, B, device=DEV)
    K.clt_rms_norm(x, w.to(DEV), 1e-5, q=q, q_scale=s, rstd=rstd)
    _, want_r, want_y = R.rms_norm(np32(hx), np64(w), 1e-5)
    b = (d / 64 + 24) * U
    assert np.all(np.abs(np64(rstd[:, -70:]) / want_r - 1) <= b)
    top = np.abs(want_y).max(-1, keepdims=True)
    assert np.all(np.abs(np64(q[:, -70:]) - 127 * want_y / top) <= 0.5 + 127 * 8 * U)
    assert not q[:, :-70].any() and torch.all(s[:, :-70] == 1.0)
    del q, s
    ws = torch.empty(K.clt_rms_norm_backward_workspace_bytes(1, B, d), dtype=torch.uint8, device=DEV)
    dw = torch.empty(1, d, device=DEV)
    K.clt_rms_norm_backward(x, w.to(DEV), rstd, dy, dy, dw, ws)
    want_dx, want_dw = R.rms_norm_backward(np32(hx), np64(w), np64(rstd[:, -70:]), np32(hg))
    size = np64(rstd[:, -70:])[..., None] * np.abs(np64(w) * np64(hg))
    size = size + np.abs(np64(hx)) * np64(rstd[:, -70:])[..., None] ** 3 * np.abs(np64(w) * np64(hg) * np64(hx)).mean(-1, keepdims=True)
    assert np.all(np.abs(np64(dy[:, -70:]) - want_dx) <= HALF["bf16"] * np.abs(want_dx) + size * b * 1.01)
    # (70 rows that are not zero: their order is all that the sum's rounding can depend on)
    assert np.all(np.abs(np64(dw) - want_dw) <= np.abs(np64(hg) * np64(hx) * np64(rstd[:, -70:])[..., None]).sum(1) * 78 * U)


def test_rms_norm_of_very_many_rows():
    """More rows than a grid has wavefronts for, eight each; and wide ones with more partial sums than a grid's second axis holds."""
    from paper_2603_21014_amd import binding as K
    B, d = (1 << 29) + 37, 8
    x, w = torch.zeros(1, B, d, dtype=torch.bfloat16, device=DEV), 1 + 0.1 * normal(1, 1, d)
    hx = normal(2, 1, 100, d).bfloat16()
    x[:, -100:] = hx.to(DEV)
    y, rstd = torch.full_like(x, 3.0), torch.empty(1, B, device=DEV)
    K.clt_rms_norm(x, w.to(DEV), 1e-5, y=y, rstd=rstd)
    _, want_r, want_y = R.rms_norm(np32(hx), np64(w), 1e-5)
    assert np.all(np.abs(np64(y[:, -100:]) - want_y) <= np.abs(want_y) * (HALF["bf16"] + 25 * U) * (1 + 2.0 ** -7))
    assert not y[:, :-100].any()
    ws = torch.empty(K.clt_rms_norm_backward_workspace_bytes(1, B, d), dtype=torch.uint8, device=DEV)
    dw = torch.empty(1, d, device=DEV)
    K.clt_rms_norm_backward(x, w.to(DEV), rstd, x, y, dw, ws)
    _, want_dw = R.rms_norm_backward(np32(hx), np64(w), np64(rstd[:, -100:]), np32(hx))
    assert np.all(np.abs(np64(dw) - want_dw) <= (np64(hx) ** 2 * np64(rstd[:, -100:])[..., None]).sum(1) * 108 * U)
    del x, y, rstd, ws
    torch.cuda.empty_cache()
    B, d = 65535 * 32 + 50, 4104
    h, dy = torch.zeros(1, B, d, device=DEV), torch.zeros(1, B, d, device=DEV)
    hx, hg, w = normal(3, 1, 40, d), normal(4, 1, 40, d), 1 + 0.1 * normal(5, 1, d)
    h[:, -40:], dy[:, -40:] = hx.to(DEV), hg.to(DEV)
    rstd = torch.ones(1, B, device=DEV)
    ws = torch.empty(K.clt_rms_norm_backward_workspace_bytes(1, B, d), dtype=torch.uint8, device=DEV)
    dw = torch.empty(1, d, device=DEV)
    K.clt_rms_norm_backward(h, w.to(DEV), rstd, dy, dy, dw, ws)
    want_dx, want_dw = R.rms_norm_backward(np32(hx), np64(w), np.ones((1, 40)), np32(hg))
    assert np.all(np.abs(np64(dw) - want_dw) <= np.abs(np64(hg) * np64(hx)).sum(1) * 48 * U)
    size = np.abs(np64(w) * np64(hg)) + np.abs(np64(hx)) * np.abs(np64(w) * np64(hg) * np64(hx)).mean(-1, keepdims=True)
    assert np.all(np.abs(np64(dy[:, -40:]) - want_dx) <= U * np.abs(want_dx) + size * (d / 64 + 24) * 1.01 * U)
    assert not dy[:, :-40].any()


def test_mx4_behind_2_to_the_32():
    from paper_2603_21014_amd import binding as K
    # a packed operand of 2^32 + ... elements, rows along the contraction and transposed
    L, rows, Kd = 5, 1 << 19, 2048
    a = torch.zeros(L, rows, Kd, dtype=torch.int8, device=DEV)
    scale = torch.ones(L, rows, device=DEV)
    ha = torch.randint(-127, 128, (1, 40, Kd), generator=torch.Generator().manual_seed(1)).to(torch.int8)
    a[-1, -40:] = ha[0].to(DEV)
    codes, scales = K.mx4_empty(L, rows, Kd, DEV)
    K.clt_mx4_quantise(a, codes, scales, a_scale=scale)
    want = R.mx4_round(np32(ha))
    got = R.mx4_unpack(codes[-1:, -4:].cpu().numpy(), scales[-1:, -1:].cpu().numpy(), 64)
    assert np.array_equal(R.mx4_values(*got)[:, -40:], R.mx4_values(*want)) and not R.mx4_values(*got)[:, :24].any()
    del a
    out = torch.empty(L, rows, Kd, dtype=torch.bfloat16, device=DEV)
    K.clt_mx4_dequantise(codes, scales, out)
    assert np.array_equal(np64(out[-1:, -40:]), R.mx4_values(*want)) and not out[-1, :-40].any()
    del out, codes, scales
    torch.cuda.empty_cache()
    # results behind the border
    M, N, Kd = 1 << 19, 8264, 64
    x, w = torch.zeros(1, M, Kd, dtype=torch.bfloat16, device=DEV), (normal(6, 1, N, Kd) / 8).to(DEV)
    hx = normal(7, 1, 50, Kd).bfloat16()
    x[:, -50:] = hx.to(DEV)
    (ac, as_), (bc, bs) = K.mx4_empty(1, M, Kd, DEV), K.mx4_empty(1, N, Kd, DEV)
    K.clt_mx4_quantise(x, ac, as_)
    K.clt_mx4_quantise(w, bc, bs)
    out = torch.full((1, M, N), 7.0, dtype=torch.bfloat16, device=DEV)
    K.clt_mx4_product(ac, as_, bc, bs, out, Kd)
    va, vw = R.mx4_values(*R.mx4_round(np32(hx)))[..., :Kd], R.mx4_values(*R.mx4_round(np32(w)))[..., :Kd]
    want = np.matmul(va, vw.transpose(0, 2, 1))
    size = np.matmul(np.abs(va), np.abs(vw).transpose(0, 2, 1))
    assert np.all(np.abs(np64(out[:, -50:]) - want) <= HALF["bf16"] * 1.01 * np.abs(want) + size * 10 * U)
    assert not out[0, :-50].any()
