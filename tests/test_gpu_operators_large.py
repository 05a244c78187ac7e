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


def test_adamw_moves_parameters_behind_2_to_the_32():
    """The parameters themselves, and a master copy of theirs: two steps against the oracle's, whose second starts from what the first stored."""
    from paper_2603_21014_amd import binding as K
    tail, n, lr, decay = 4099, FAR + 4099, 1e-2, 0.5
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device=DEV)
    hp, hg = normal(11, tail), (1e-3 * normal(12, tail)).bfloat16()
    for with_master in (False, True):
        p, g, m, v = z(torch.bfloat16), z(torch.bfloat16), z(torch.uint8), z(torch.uint8)
        ms, vs = z(torch.uint8, (n + 127) // 128), z(torch.uint8, (n + 127) // 128)
        master = z(torch.float32) if with_master else None
        p[FAR:], g[FAR:] = hp.to(DEV), hg.to(DEV)
        if with_master:
            master[FAR:] = hp.to(DEV)
        opt = K.AdamW([K.AdamWTensor(p, g, m, v, ms, vs, master, decay)], seed=5)
        w = np32(hp) if with_master else np32(hp.bfloat16())
        blocks = -(-tail // 128)
        state = [np.zeros(tail, np.uint8), np.zeros(tail, np.uint8), np.zeros(blocks, np.uint8), np.zeros(blocks, np.uint8)]
        real = R.random_bits
        try:
            R.random_bits = lambda seed, t, index, k: real(seed, t, index, k, first=FAR)
            for t in (1, 2):
                opt.step(t, lr)
                torch.cuda.synchronize()
                o = R.adamw(w, np32(hg), state[0], state[1], t, lr, 0.9, 0.999, 1e-8, decay, state[2], state[3], 5, 0)
                state = [o["m"], o["v"], o["m_scale"], o["v_scale"]]
                # as of small tensors: update of square root, reciprocal and four products, product with 1 - lr decay, addition
                bound = np.abs(w * (1.0 - lr * decay) - o["p"]) * 16 * U + np.abs(w) * 3 * U + 1e-38
                moved = np.abs(o["p"] - w)
                if with_master:
                    got = np64(master[FAR:])
                    assert np.all(np.abs(got - o["p"]) <= bound) and torch.equal(p[FAR:], master[FAR:].bfloat16())
                    assert (moved > 2 * bound).mean() > 0.99      # (or the comparison above would say nothing)
                    w = np32(master[FAR:])
                else:
                    got = np64(p[FAR:])
                    assert np.all(np.abs(got - o["p"]) <= 2 * bound + HALF["bf16"] * np.abs(o["p"]) * 1.01)
                    assert (moved > 2 * (2 * bound + HALF["bf16"] * np.abs(o["p"]))).mean() > 0.5
                    w = np32(p[FAR:])
        finally:
            R.random_bits = real
        assert not p[:FAR].any() and (master is None or not master[:FAR].any())
        del p, g, m, v, ms, vs, master, opt
        torch.cuda.empty_cache()


def test_mx4_transposed_behind_2_to_the_32():
    """A matrix of more than 2^32 elements whose columns are packed; both types."""
    from paper_2603_21014_amd import binding as K
    for dtype, L, rows, Kd in ((torch.bfloat16, 3, 1 << 20, 1416), (torch.float32, 2, (1 << 20) - 8, 2056)):
        assert L * rows * Kd > FAR
        a = torch.zeros(L, Kd, rows, dtype=dtype, device=DEV)
        ha = (normal(21, 1, 72, Kd) * torch.exp(normal(22, 1, 72, 1))).to(dtype)
        a[-1, :, -72:] = ha[0].T.contiguous().to(DEV)
        codes, scales = K.mx4_empty(L, rows, Kd, DEV)
        K.clt_mx4_quantise(a, codes, scales, transposed=True)
        del a
        first = (rows - 72) // 64      # the panels that hold the last 72 rows
        got = R.mx4_unpack(codes[-1:, 4 * first:].cpu().numpy(), scales[-1:, first:].cpu().numpy(), rows - 64 * first)
        want = R.mx4_round(np32(ha))
        assert np.array_equal(R.mx4_values(*got)[:, -72:], R.mx4_values(*want)) and not R.mx4_values(*got)[:, :-72].any()
        out = torch.full((L, rows, Kd), 3.0, dtype=dtype, device=DEV)
        K.clt_mx4_dequantise(codes, scales, out)
        assert np.array_equal(np64(out[-1:, -72:]), R.mx4_values(*want)[..., :Kd]) and not out[-1, :-72].any() and not out[0].any()
        del codes, scales, out
        torch.cuda.empty_cache()


def _far_blocks(L, rows, KS, seed):
    """(codes, packed codes, packed scales) of [L, rows, 128 KS]: small numbers in eight steps (the first, the last, around every sixth between), zeros
    elsewhere; the codes of those steps as [L, rows, 8 * 128], their scales 2^-1, 1 or 2."""
    steps = sorted({0, 1, KS // 5, KS // 3, KS // 2, KS - 1000, KS - 2, KS - 1})
    g = np.random.default_rng(seed)
    codes, s = g.integers(0, 16, (L, rows, 1024)).astype(np.uint8), g.integers(126, 129, (L, rows, 32)).astype(np.uint8)
    pc, ps = R.mx4_pack(codes, s)
    panels = (rows + 63) // 64
    dc = torch.zeros(L, 4 * panels, KS, 1024, dtype=torch.uint8, device=DEV)
    ds = torch.full((L, panels, KS, 256), 127, dtype=torch.uint8, device=DEV)
    dc[:, :, steps], ds[:, :, steps] = torch.from_numpy(pc).to(DEV), torch.from_numpy(ps).to(DEV)
    return R.mx4_values(codes, s), dc, ds


def test_mx4_longest_contractions():
    """K = 2^22, the longest that is taken: every product kernel, packing and unpacking.  The numbers are multiples of 2^-4 below 2^18 in sum, so
    every order of the sum is exact."""
    from paper_2603_21014_amd import binding as K
    KS, Kd = 1 << 15, 1 << 22
    # one tile of tokens; two, and more than one panel of features; the tile kernel (160 tiles)
    for L, M, N in ((1, 1, 72), (1, 40, 72), (160, 40, 8)):
        va, ac, as_ = _far_blocks(L, M, KS, 31)
        vb, bc, bs = _far_blocks(L, N, KS, 32)
        want = np.matmul(va, vb.transpose(0, 2, 1))
        for dtype in (torch.float32, torch.bfloat16):
            out = torch.full((L, M, N), 9.0, dtype=dtype, device=DEV)
            K.clt_mx4_product(ac, as_, bc, bs, out, Kd)
            assert torch.equal(out.cpu(), torch.from_numpy(want).to(dtype)), (L, M, N)
        del ac, as_, bc, bs
        torch.cuda.empty_cache()
    rows, last = 70, 4096
    for transposed in (False, True):
        rows = 72 if transposed else 70
        x = torch.zeros(1, rows, Kd, dtype=torch.bfloat16, device=DEV)
        hx = normal(33, 1, rows, last).bfloat16()
        x[:, :, -last:] = hx.to(DEV)
        x = x.transpose(1, 2).contiguous() if transposed else x
        codes, scales = K.mx4_empty(1, rows, Kd, DEV)
        K.clt_mx4_quantise(x, codes, scales, transposed=transposed)
        del x
        n = last // 128
        got = R.mx4_unpack(codes[:, :, -n:].cpu().numpy(), scales[:, :, -n:].cpu().numpy(), rows)
        want = R.mx4_values(*R.mx4_round(np32(hx)))
        assert np.array_equal(R.mx4_values(*got), want)
        out = torch.empty(1, rows, Kd, dtype=torch.bfloat16, device=DEV)
        K.clt_mx4_dequantise(codes, scales, out)
        assert np.array_equal(np64(out[:, :, -last:]), want) and not out[:, :, :-last].any()
        del codes, scales, out
        torch.cuda.empty_cache()
