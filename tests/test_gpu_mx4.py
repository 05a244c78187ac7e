"""4-bit microscaled floating point: packing (bit for bit), unpacking and the product, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as R
from operators_testlib import DEV, HALF, T, U, Guarded, normal, np32, np64, replayed

pytestmark = pytest.mark.gpu

# (L, rows, K): one row; K below, at and around a block of 32 and a step of 128; rows around 16 and a panel of 64
PACKS = [(1, 1, 8), (2, 3, 32), (1, 16, 40), (3, 17, 128), (1, 63, 136), (2, 64, 256), (1, 65, 264), (2, 200, 520), (1, 24, 2056), (1, 1000, 768), (2, 256, 1024)]


def matrix(L, rows, K, dtype, seed=0):
    x = normal(seed + 1, L, rows, K) * torch.exp(normal(seed + 2, L, rows, 1))
    x[:, ::7, : K // 2] *= 2.0 ** -20
    x[:, rows // 2] = 0.0
    return x.to(T[dtype])


def pack_room(K_, L, rows, K):
    c, s = K_.mx4_empty(L, rows, K, DEV)
    return Guarded(c.shape, torch.uint8, torch.full_like(c, 0x5A)), Guarded(s.shape, torch.uint8, torch.full_like(s, 0x5A))


def check_pack(codes, scales, want_codes, want_scales, rows):
    gc, gs = R.mx4_unpack(codes.t.cpu().numpy(), scales.t.cpu().numpy(), rows)
    assert np.array_equal(gs, want_scales)
    # (a zero may carry either sign: it stands for the same value)
    assert np.array_equal(np.where((gc & 7) == 0, 0, gc), np.where((want_codes & 7) == 0, 0, want_codes))
    codes.check()
    scales.check()


@pytest.mark.parametrize("L,rows,K", PACKS)
@pytest.mark.parametrize("kind", ["bf16", "f32", "int8", "bf16 transposed", "f32 transposed"])
def test_packing(kind, L, rows, K):
    from paper_2603_21014_amd import binding as B
    transposed = "transposed" in kind
    if transposed:
        rows = -(-rows // 8) * 8
    codes, scales = pack_room(B, L, rows, K)
    a_scale = None
    if kind == "int8":
        a = torch.randint(-127, 128, (L, rows, K), generator=torch.Generator().manual_seed(5)).to(torch.int8)
        a_scale = torch.exp(normal(6, L, rows))
        values = np32(a) * np32(a_scale)[..., None]
        B.clt_mx4_quantise(a.to(DEV), codes.t, scales.t, a_scale=a_scale.to(DEV))
    else:
        a = matrix(L, rows, K, kind[:4].strip())
        values = np32(a)
        a = a.transpose(1, 2).contiguous() if transposed else a
        B.clt_mx4_quantise(a.to(DEV), codes.t, scales.t, transposed=transposed)
    torch.cuda.synchronize()
    want_codes, want_scales = R.mx4_round(values)
    check_pack(codes, scales, want_codes, want_scales, rows)
    pc, ps = R.mx4_pack(np.full_like(want_codes, 15), np.full_like(want_scales, 255))      # where something belongs
    assert np.all(codes.t.cpu().numpy()[pc == 0] == 0x5A) and np.all(scales.t.cpu().numpy()[ps == 0] == 0x5A), "rows beyond the last one were written"
    for dtype in ("bf16", "f32"):
        out = Guarded((L, rows, K), T[dtype])
        B.clt_mx4_dequantise(codes.t, scales.t, out.t)
        torch.cuda.synchronize()
        assert np.array_equal(np64(out.t), R.mx4_values(want_codes, want_scales)[..., :K])
        out.check()


def test_special_values():
    """The types' smallest and largest numbers, ties, infinities and NaN, in blocks of their own."""
    from paper_2603_21014_amd import binding as B
    x = np.zeros((1, 10, 64), np.float32)
    x[0, 0, :8] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5]
    x[0, 1, :4] = [7, 6.999, -7, 3.5]                         # the largest reaches 1.75 * 4: the next power
    x[0, 2, :3] = [1e-45, -3e-45, 2e-42]                      # denormals
    x[0, 3, :3] = [3.4e38, -1e38, 1e37]
    x[0, 4, 3] = np.inf
    x[0, 5, 40] = -np.inf
    x[0, 6, 33] = np.nan
    x[0, 7] = -0.0
    x[0, 8, :3] = [2.0 ** -126, 2.0 ** -127, 2.0 ** -128]
    x[0, 9, ::2] = 2.0 ** -65
    for transposed in (False, True):
        rows = 16 if transposed else 10
        v = np.zeros((1, rows, 64), np.float32)
        v[:, :10] = x
        codes, scales = pack_room(B, 1, rows, 64)
        a = torch.from_numpy(v).transpose(1, 2).contiguous() if transposed else torch.from_numpy(v)
        B.clt_mx4_quantise(a.to(DEV), codes.t, scales.t, transposed=transposed)
        torch.cuda.synchronize()
        want = R.mx4_round(v)
        check_pack(codes, scales, *want, rows)
        out = torch.empty(1, rows, 64, device=DEV)
        B.clt_mx4_dequantise(codes.t, scales.t, out)
        with np.errstate(over="ignore"):      # 3.4e38 rounds to 4 * 2^126 = 2^128, which fp32 holds as an infinity
            got, ref = np32(out), R.mx4_values(*want)[..., :64].astype(np.float32)
        assert np.isposinf(ref[0, 3, 0]) and np.isfinite(ref[0, 3, 1:]).all()
        assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.isnan(got[0, 4, :32]).all() and not np.isnan(got[0, 4, 32:]).any()
        assert np.array_equal(got[~np.isnan(ref)], ref[~np.isnan(ref)])


# (L, M, N, K): single tokens, few rows, odd batches, one and many steps, tiles that end inside a panel, several layers
PRODUCTS = [(1, 1, 8, 8), (1, 1, 256, 2048), (16, 1, 512, 136), (3, 2, 72, 64), (1, 7, 264, 520), (2, 16, 128, 128), (1, 17, 1000, 264), (2, 33, 520, 768), (1, 64, 64, 256),
            (1, 65, 2056, 136), (3, 100, 256, 264), (1, 128, 256, 512), (1, 200, 776, 2056), (2, 255, 512, 384), (1, 256, 1024, 1024), (1, 300, 520, 1160), (1, 513, 264, 4096),
            (1, 1030, 1288, 640), (4, 260, 264, 128)]


def operands(B, L, M, N, K, seed=0):
    a, w = matrix(L, M, K, "bf16", seed), (normal(seed + 9, L, N, K) / K ** 0.5)
    (ac, as_), (bc, bs) = B.mx4_empty(L, M, K, DEV), B.mx4_empty(L, N, K, DEV)
    for t in (ac, as_, bc, bs):      # rows beyond the last hold anything, scales that are NaN among it
        t.fill_(255)
    B.clt_mx4_quantise(a.to(DEV), ac, as_)
    B.clt_mx4_quantise(w.transpose(1, 2).contiguous().to(DEV) if N % 8 == 0 else None, bc, bs, transposed=True)
    va, vw = R.mx4_values(*R.mx4_round(np32(a)))[..., :K], R.mx4_values(*R.mx4_round(np32(w)))[..., :K]
    return (ac, as_, bc, bs), va, vw


def check_product(out, va, vw, bias, theta, dtype):
    want = np.matmul(va, vw.transpose(0, 2, 1)) + (0 if bias is None else np64(bias)[:, None, :])
    # partial sums in fp32 in any order and grouping, and the bias
    size = np.matmul(np.abs(va), np.abs(vw).transpose(0, 2, 1)) + (0 if bias is None else np.abs(np64(bias))[:, None, :])
    err = size * (va.shape[-1] / 32 + 8) * U
    got = np64(out)
    if theta is None:
        assert np.all(np.abs(got - want) <= err + HALF[dtype] * np.abs(want) * 1.01 + 1e-38)
        return
    th = np64(theta)[:, None, :]
    kept = np.abs(got - want) <= err + HALF[dtype] * np.abs(want) * 1.01 + 1e-38
    assert np.all(np.where(want > th + err, kept, np.where(want <= th - err, got == 0, kept | (got == 0))))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,M,N,K", PRODUCTS)
def test_product(dtype, L, M, N, K):
    from paper_2603_21014_amd import binding as B
    packed, va, vw = operands(B, L, M, N, K)
    bias, theta = 0.1 * normal(30, L, N), 0.2 + 0.1 * normal(31, L, N)
    for b, t in ((None, None), (bias, theta), (bias, None), (None, theta)):
        out = Guarded((L, M, N), T[dtype])
        B.clt_mx4_product(*packed, out.t, K, bias=None if b is None else b.to(DEV), theta=None if t is None else t.to(DEV))
        torch.cuda.synchronize()
        check_product(out.t, va, vw, b, t, dtype)
        out.check()


# Where tiles of 128 tokens by 256 features are enough for the chip (160 and more): one step and many, fewer tiles than workgroups, as many, and
# several to each; tokens, features and tile groups that end early
TILED = [(160, 33, 8, 8), (83, 130, 264, 128), (300, 129, 264, 136), (1, 2600, 2056, 264), (2, 1700, 4104, 392), (1, 5000, 4104, 136), (20, 1000, 264, 4104), (700, 65, 40, 256),
         (5, 1030, 1288, 640), (512, 128, 256, 128), (1, 20488, 24, 384),
         # four tiles and more to a workgroup, of one step, a few, around eight and twenty; and of more
         (2100, 33, 8, 8), (520, 130, 264, 136), (2050, 65, 24, 384), (2048, 40, 72, 896), (2060, 33, 16, 1032), (2060, 40, 24, 2560), (2060, 40, 24, 2568), (3, 20000, 1288, 72)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L,M,N,K", TILED)
def test_product_of_many_tiles(dtype, L, M, N, K):
    """In 64 bits on the device, on the values that unpacking gives (bit for bit the oracle's, above)."""
    from paper_2603_21014_amd import binding as B
    assert M > 32 and L * -(-M // 128) * -(-N // 256) >= 160
    g = torch.Generator(device=DEV).manual_seed(M + K)
    packed, values = [], []
    for rows in (M, N):
        c, sc = B.mx4_empty(L, rows, K, DEV)
        c.fill_(255), sc.fill_(255)      # rows beyond the last hold anything
        x = torch.randn(L, rows, K, generator=g, device=DEV)
        B.clt_mx4_quantise(x, c, sc)
        B.clt_mx4_dequantise(c, sc, x)
        packed += [c, sc]
        values.append(x.double())
    va, vw = values[0], values[1].transpose(1, 2).contiguous()
    exact, size = torch.matmul(va, vw), torch.matmul(va.abs(), vw.abs())
    bias, theta = (torch.randn(L, N, generator=g, device=DEV) for _ in range(2))
    for b, th in ((None, None), (bias, theta), (bias, None), (None, theta)):
        out = Guarded((L, M, N), T[dtype])
        B.clt_mx4_product(*packed, out.t, K, bias=b, theta=th)
        got, want, err = out.t.double(), exact, size
        if b is not None:
            want, err = exact + b.double()[:, None], size + b.double().abs()[:, None]
        err = err * ((K / 32 + 8) * U)      # partial sums in fp32 in any order and grouping, and the bias
        right = (got - want).abs() <= err + HALF[dtype] * 1.01 * want.abs()
        if th is not None:
            t = th.double()[:, None]
            right = torch.where(want > t + err, right, torch.where(want <= t - err, got == 0, right | (got == 0)))
        assert right.all()
        out.check()


def test_product_of_broken_blocks():
    """A block with a NaN makes its row (or column) NaN and no other; with a threshold NaN is not above it."""
    from paper_2603_21014_amd import binding as B
    for M, K in ((3, 264), (150, 264), (20600, 264), (262000, 136)):
        L, N = 1, 72
        a, w = matrix(L, M, K, "bf16"), normal(9, L, N, K)
        a[0, 2, K - 64], w[0, 11, 3] = float("nan"), float("inf")
        (ac, as_), (bc, bs) = B.mx4_empty(L, M, K, DEV), B.mx4_empty(L, N, K, DEV)
        B.clt_mx4_quantise(a.to(DEV), ac, as_)
        B.clt_mx4_quantise(w.to(DEV), bc, bs)
        for dtype in ("f32", "bf16"):
            out = torch.empty(L, M, N, device=DEV, dtype=T[dtype])
            B.clt_mx4_product(ac, as_, bc, bs, out, K)
            nan = torch.isnan(out.cpu())[0]
            want = torch.zeros(M, N, dtype=torch.bool)
            want[2], want[:, 11] = True, True
            assert torch.equal(nan, want)
            B.clt_mx4_product(ac, as_, bc, bs, out, K, theta=torch.full((L, N), -1e30, device=DEV))
            assert not out.cpu()[0][want].any() and not torch.isnan(out).any()


def test_product_of_exact_numbers_is_exact():
    """Small whole numbers with one scale: every partial sum is a number that fp32 holds, so the order of the sum cannot matter."""
    from paper_2603_21014_amd import binding as B
    for L, M, N, K in ((2, 16, 264, 1000), (2, 300, 264, 1000), (50, 300, 264, 1000), (7, 1100, 1032, 520), (400, 300, 264, 200)):
        g = torch.Generator().manual_seed(3)
        a, w = (torch.randint(-4, 5, s, generator=g).float() for s in ((L, M, K), (L, N, K)))
        a[:, :, ::32], w[:, :, ::32] = 4.0, -4.0
        (ac, as_), (bc, bs) = B.mx4_empty(L, M, K, DEV), B.mx4_empty(L, N, K, DEV)
        B.clt_mx4_quantise(a.to(DEV), ac, as_)
        B.clt_mx4_quantise(w.to(DEV), bc, bs)
        exact = torch.matmul(a.double(), w.double().transpose(1, 2).contiguous())
        for dtype in ("f32", "bf16"):
            out = torch.empty(L, M, N, device=DEV, dtype=T[dtype])
            B.clt_mx4_product(ac, as_, bc, bs, out, K)
            assert torch.equal(out.cpu(), exact.to(T[dtype]))


def test_streams_and_graphs():
    from paper_2603_21014_amd import binding as B
    for L, M in ((2, 1), (2, 40), (2, 300), (30, 200), (90, 200), (400, 200)):
        N, K = 520, 776
        x, w = matrix(L, M, K, "bf16").to(DEV), (normal(8, L, K, N) / K ** 0.5).to(DEV)
        (ac, as_), (bc, bs) = B.mx4_empty(L, M, K, DEV), B.mx4_empty(L, N, K, DEV)
        out = torch.empty(L, M, N, dtype=torch.bfloat16, device=DEV)

        def call():
            B.clt_mx4_quantise(w, bc, bs, transposed=True)
            B.clt_mx4_quantise(x, ac, as_)
            B.clt_mx4_product(ac, as_, bc, bs, out, K)
        call()
        want = out.clone()
        for got in replayed(call, (out, ac, bc)):
            assert torch.equal(got[0], want)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            call()
        s.synchronize()
        assert torch.equal(out, want)


def test_binding_refusals_on_the_device():
    from paper_2603_21014_amd import binding as B
    c, s = B.mx4_empty(2, 24, 64, DEV)
    x = torch.zeros(2, 24, 64, device=DEV)
    out = torch.full((2, 24, 24), 3.0, device=DEV)
    for bad in (lambda: B.clt_mx4_quantise(x, c[:1], s), lambda: B.clt_mx4_quantise(x, c, s[:, :, :, :128]), lambda: B.clt_mx4_quantise(x.transpose(1, 2), c, s),
                lambda: B.clt_mx4_quantise(x.to(torch.int8), c, s, a_scale=x[..., :2]), lambda: B.clt_mx4_dequantise(c, s, x[:1]),
                lambda: B.clt_mx4_product(c, s, c, s, out, 192), lambda: B.clt_mx4_product(c, s, c, s, out.half(), 64),
                lambda: B.clt_mx4_product(c, s, c, s, out, 64, bias=out)):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: B.mx4_empty(1, 0, 64, DEV), lambda: B.clt_mx4_quantise(x.to(torch.int8), c, s)):
        with pytest.raises(B.CLTError):
            bad()
    torch.cuda.synchronize()
    assert torch.all(out == 3.0)
